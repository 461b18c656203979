"""Attention over the stored history, drafted trees, accumulated weights and eviction
on the GPU, against the 64-bit forms of history_ref with their error bounds."""
import sys

import numpy as np
import pytest

import history_ref as R
import workloads as W

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_02780_amd  # noqa: F401  (fails loudly without the built library)


def log(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda().view(torch.bfloat16)


def host(t):
    return t.contiguous().view(torch.int16).cpu().numpy()


def bf(rng, *shape, scale=1.0):
    return W.bf16_bits(rng.standard_normal(shape).astype(np.float32) * scale)


class Stream:
    """An index that keeps values, and the same rows on the host."""

    def __init__(self, rng, heads, runs, L=1, extra=7, n_recent=0, scale=1.0):
        import paper_2609_02780_amd as P
        self.Hq, self.Hk, self.d = heads
        self.L = L
        self.rows = [t for f, t in runs for _ in range(f)]
        F, n = len(self.rows), sum(self.rows)
        self.ix = P.ShallowIndex(L, *heads, F + 3, n + extra, n_recent=n_recent)
        self.ix.attach_values()
        self.ix.arena.fill_(255)              # what no append wrote is NaN
        self.ix.value_arena.fill_(255)
        self.k = [np.zeros((self.Hk, 0, self.d), np.uint16) for _ in range(L)]
        self.v = [np.zeros((self.Hk, 0, self.d), np.uint16) for _ in range(L)]
        for f, t in runs:
            ks = [bf(rng, self.Hk, f * t, self.d, scale=scale) for _ in range(L)]
            vs = [bf(rng, self.Hk, f * t, self.d) for _ in range(L)]
            self.ix.append_kv([dev(x) for x in ks], [dev(x) for x in vs], f, t)
            self.k = [np.concatenate([a, b], 1) for a, b in zip(self.k, ks)]
            self.v = [np.concatenate([a, b], 1) for a, b in zip(self.v, vs)]

    @property
    def frame(self):
        return np.repeat(np.arange(len(self.rows)), self.rows)

    def seen(self, layer, frames=None, first=0):
        f = self.frame
        keep = f >= first
        if frames is not None:
            keep &= np.isin(f, [x for x in frames if first <= x < len(self.rows)])
        return (R.f64(self.k[layer])[:, keep], R.f64(self.v[layer])[:, keep], keep,
                (len(self.rows) - f[keep]).astype(np.float64))


class Own:
    def __init__(self, rng, heads, n, room=3):
        _, Hk, d = heads
        self.k, self.v, self.n = bf(rng, Hk, n + room, d), bf(rng, Hk, n + room, d), n
        self.k[:, n:] = 0x7FC0                 # NaN behind the last token
        self.v[:, n:] = 0x7FC0
        self.arg = (dev(self.k), dev(self.v), n)


def want(st, layer, q, own=None, parents=None, frames=None, first=0, softcap=0.0, slopes=None):
    k, v, _, age = st.seen(layer, frames, first)
    nq = q.shape[1]
    mask = np.ones((nq, k.shape[1]), dtype=bool)
    if own is not None:
        k = np.concatenate([k, R.f64(own.k[:, :own.n])], 1)
        v = np.concatenate([v, R.f64(own.v[:, :own.n])], 1)
        age = np.concatenate([age, np.zeros(own.n)])
        mask = np.concatenate([mask, R.causal(nq, own.n) if parents is None else R.tree_mask(parents, own.n)], 1)
    return R.attend(R.f64(q), k, v, mask, st.Hq // st.Hk, softcap, slopes, age)


def check(got, ref, what=""):
    out, lse = got
    o, z, bo, bz = ref
    g = R.f64(host(out))
    assert np.isfinite(g).all(), what
    bad = np.abs(g - o) > bo
    assert not bad.any(), (what, "out", int(bad.sum()), float(np.abs(g - o).max()), float((np.abs(g - o) / bo).max()))
    y = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(y), np.isneginf(z)), (what, "lse of empty rows")
    live = ~np.isneginf(z)
    bad = np.abs(y[live] - z[live]) > bz[live]
    assert not bad.any(), (what, "lse", int(bad.sum()), float(np.abs(y[live] - z[live]).max()))


HEADS = [(4, 2, 64), (28, 4, 128), (3, 1, 64), (16, 1, 128), (8, 8, 64), (2, 2, 128)]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("nq,runs,text", [
    (1, [(1, 1)], None), (1, [(40, 49)], 0), (1, [(3, 127), (9, 16)], 6), (2, [(1, 129)], 300), (5, [(64, 16)], None),
    (17, [(7, 33)], 1), (33, [(11, 30), (4, 7)], 0), (70, [(5, 64)], 62), (130, [(2, 5)], 0), (300, [(13, 20)], 9),
], ids=str)
def test_attend(heads, nq, runs, text):
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], heads[2], nq, len(runs)])
    st = Stream(rng, heads, runs, L=2)
    q = bf(rng, heads[0], nq, heads[2], scale=1.5)
    own = Own(rng, heads, text + nq) if text is not None else None
    slopes = np.linspace(-0.02, 0.3, heads[0]).astype(np.float32)
    some = [0, len(st.rows) - 1, -1, 0, 10 ** 12, len(st.rows) // 2]
    for layer, softcap, sl, frames in ((1, 0.0, None, None), (0, 4.0, None, None), (1, 0.0, slopes, None),
                                       (0, 20.0, slopes, some), (1, 0.0, None, some)):
        log("case", heads, nq, runs, text, layer, softcap, sl is not None, frames is not None)
        att = P.HistoryAttention([st.ix], softcap, None if sl is None else torch.from_numpy(sl).cuda())
        fr = None if frames is None else torch.tensor([frames], device="cuda")
        out, lse = att(layer, [dev(q)], own=None if own is None else [own.arg], frames=fr)
        ref = want(st, layer, q, own, None, frames, 0, softcap, None if sl is None else sl.astype(np.float64))
        check((out[0], lse[0]), ref, (layer, softcap, frames))


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (16, 1, 128)], ids=str)
@pytest.mark.parametrize("n,text,runs", [(1, 0, [(3, 5)]), (8, 100, [(20, 16)]), (31, 1, [(1, 1)]), (64, 33, [(30, 49)]),
                                         (200, 65, [(4, 100)]), (512, 0, [(2, 64)])], ids=str)
def test_tree(heads, n, text, runs):
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], n, text])
    st = Stream(rng, heads, runs)
    q = bf(rng, heads[0], n, heads[2], scale=1.5)
    own = Own(rng, heads, text + n)
    att = P.HistoryAttention([st.ix])
    wild = np.array([rng.integers(-1, i) if i else -1 for i in range(n)], dtype=np.int32)
    shapes = {"random": wild, "star": np.full(n, -1, np.int32), "chain": np.arange(n, dtype=np.int32) - 1,
              "bushy": np.array([-1 if i == 0 else (i - 1) // 3 for i in range(n)], dtype=np.int32)}
    shapes["wrong parents are roots"] = np.where(np.arange(n) % 3 == 2, np.arange(n) + 5, shapes["bushy"]).astype(np.int32)
    for name, par in shapes.items():
        log("case", heads, n, text, name)
        out, lse = att(0, [dev(q)], own=[own.arg], tree=[torch.from_numpy(par).cuda()])
        check((out[0], lse[0]), want(st, 0, q, own, par), name)
    out, lse = att(0, [dev(q)], own=[own.arg], tree=[torch.from_numpy(shapes["chain"]).cuda()])
    flat, flse = att(0, [dev(q)], own=[own.arg])
    assert torch.equal(out[0], flat[0]) and torch.equal(lse[0], flse[0])     # a chain is the causal mask


def test_nothing_to_see():
    """An empty index, a list of nothing, and the own tokens alone."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(5)
    heads = (6, 2, 64)
    empty = P.ShallowIndex(1, *heads, 4, 16)
    empty.attach_values()
    q = bf(rng, 6, 9, 64)
    out, lse = P.HistoryAttention([empty])(0, [dev(q)])
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    st = Stream(rng, heads, [(5, 20)])
    att = P.HistoryAttention([st.ix], slopes=torch.zeros(6, device="cuda"))
    nothing = torch.tensor([[-1, 99, -7, 5]], device="cuda")
    out, lse = att(0, [dev(q)], frames=nothing)
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    kinds = torch.ones((1, 2), dtype=torch.int32, device="cuda")
    out, lse = att(0, [dev(q)], frames=torch.tensor([[1, 2]], device="cuda"), kinds=kinds)
    assert not out[0].any() and torch.isneginf(lse[0]).all()
    own = Own(rng, heads, 12)
    for a, fr in ((att, nothing), (P.HistoryAttention([empty]), None)):
        out, lse = a(0, [dev(q)], own=[own.arg], frames=fr)
        check((out[0], lse[0]), want(st, 0, q, own, None, []))
    st.ix.weights.fill_(3.0)
    att.accumulate(0, [dev(q)], [torch.full((6, 9), float("-inf"), device="cuda")])
    assert torch.equal(st.ix.weights, torch.full_like(st.ix.weights, 3.0))     # nothing seen, nothing added
    att.accumulate(0, [dev(q)], [torch.zeros(6, 9, device="cuda")], frames=nothing, decay=0.5)
    assert torch.equal(st.ix.weights, torch.full_like(st.ix.weights, 1.5))
    P.HistoryAttention([empty]).accumulate(0, [dev(q)], [torch.zeros(6, 9, device="cuda")], decay=0.0)
    torch.cuda.synchronize()


@pytest.mark.parametrize("nq", [1, 6, 90])
def test_ragged_batch(nq):
    """More streams than one launch takes, of many lengths (one empty), each with its own mask."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(nq)
    heads = (8, 2, 64)
    sts = [Stream(rng, heads, [(1 + 7 * (s % 5), 1 + 11 * s)]) for s in range(18)]
    qs = [bf(rng, 8, nq + s % 3, 64, scale=1.5) for s in range(18)]
    owns = [None if s % 4 == 1 else Own(rng, heads, nq + s % 3 + 5 * s, room=s) for s in range(18)]
    pars = [torch.tensor([i - 1 if i % 4 else -1 for i in range(qs[s].shape[1])], dtype=torch.int32, device="cuda")
            if s % 4 == 2 else None for s in range(18)]
    lists = torch.tensor([[s % 3, -1, 4, 4, 30] for s in range(18)], device="cuda")
    att = P.HistoryAttention([s.ix for s in sts], 15.0)
    for fr in (None, lists):
        out, lse = att(0, [dev(q) for q in qs], own=[o and o.arg for o in owns], tree=pars, frames=fr)
        for s in range(18):
            log("stream", s, fr is not None)
            ref = want(sts[s], 0, qs[s], owns[s], None if pars[s] is None else pars[s].cpu().numpy(),
                       None if fr is None else fr[s].tolist(), 0, 15.0)
            check((out[s], lse[s]), ref, s)
    # one index for several streams of a call
    two = P.HistoryAttention([sts[3].ix, sts[3].ix])
    out, lse = two(0, [dev(qs[0]), dev(qs[5])])
    for o, z, q in zip(out, lse, (qs[0], qs[5])):
        check((o, z), want(sts[3], 0, q))


def test_long_history():
    """Rows enough for many shares, one query far above the rest at the very end and start."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(11)
    heads = (4, 2, 128)
    st = Stream(rng, heads, [(500, 61), (1, 3)])
    n = st.k[0].shape[1]
    for nq in (1, 40, 150):
        q = bf(rng, 4, nq, 128)
        q[0, 0] = W.bf16_bits(R.f64(st.k[0][0, 0]).astype(np.float32) * 3)       # its score: about 34
        q[1, 0] = W.bf16_bits(R.f64(st.k[0][0, n - 1]).astype(np.float32) * 3)
        log("n_q", nq)
        out, lse = P.HistoryAttention([st.ix])(0, [dev(q)])
        check((out[0], lse[0]), want(st, 0, q), nq)


def test_large_scores():
    """Scores of some hundreds, of both signs, and a cap far below them."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(12)
    st = Stream(rng, (4, 2, 64), [(9, 70)], scale=12.0)
    q = bf(rng, 4, 20, 64, scale=12.0)
    for cap in (0.0, 30.0, 0.01, 1e6):
        out, lse = P.HistoryAttention([st.ix], cap)(0, [dev(q)])
        check((out[0], lse[0]), want(st, 0, q, softcap=cap), cap)


@pytest.mark.parametrize("rows", [1, 2, 3, 31, 32, 33, 127, 700])
def test_bias_over_equal_frames(rows):
    """Ages from the frames' one size, and (with a list, or wide questions) from the map."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(rows)
    heads = (8, 2, 64)
    st = Stream(rng, heads, [(max(2, 900 // rows), rows)])
    slopes = np.linspace(-0.05, 0.4, 8).astype(np.float32)
    att = P.HistoryAttention([st.ix], 9.0, torch.from_numpy(slopes).cuda())
    every = torch.arange(len(st.rows), device="cuda")[None]
    for nq in (1, 10, 20, 40):
        q = bf(rng, 8, nq, 64, scale=1.5)
        own = Own(rng, heads, nq + 3)
        log("rows", rows, "n_q", nq)
        ref = want(st, 0, q, own, softcap=9.0, slopes=slopes.astype(np.float64))
        for fr in (None, every):
            out, lse = att(0, [dev(q)], own=[own.arg], frames=fr)
            check((out[0], lse[0]), ref, (rows, nq))
            att.accumulate(0, [dev(q)], lse, frames=fr, decay=0.0)
            k, _, _, age = st.seen(0)
            w, b = R.weights(R.f64(q), k, lse[0].cpu().numpy(), 4, 9.0, slopes.astype(np.float64), age)
            assert (np.abs(st.ix.weights[0].double().cpu().numpy() - w) <= b).all()


def test_far_addresses():
    """Rows whose places lie beyond 2^32 bytes of the arenas, in every operator."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(15)
    heads, rows = (16, 8, 128), 1_300_000                  # a KV head: 333 MB, a layer: 2.7 GB
    ix = P.ShallowIndex(2, *heads, 40, rows)
    ix.attach_values()
    st = Stream(rng, heads, [], L=2)
    st.ix, st.rows = ix, [33] * 20
    st.k = [bf(rng, 8, 660, 128) for _ in range(2)]
    st.v = [bf(rng, 8, 660, 128) for _ in range(2)]
    ix.append_kv([dev(x) for x in st.k], [dev(x) for x in st.v], 20, 33)
    q = bf(rng, 16, 5, 128)
    lists = torch.tensor([[19, 3, 7]], device="cuda")
    for att, fr in ((P.HistoryAttention([ix]), None), (P.HistoryAttention([ix]), lists)):
        out, lse = att(1, [dev(q)], frames=fr)
        check((out[0], lse[0]), want(st, 1, q, frames=None if fr is None else fr[0].tolist()))
        att.accumulate(1, [dev(q)], lse, frames=fr, decay=0.0)
        k, _, keep, _ = st.seen(1, None if fr is None else fr[0].tolist())
        w, b = R.weights(R.f64(q), k, lse[0].cpu().numpy(), 2)
        got = ix.weights[1].double().cpu().numpy()
        assert (np.abs(got[:, keep] - w) <= b).all() and not got[:, ~keep].any()
    dst = P.ShallowIndex(2, *heads, 40, rows)
    dst.attach_values()
    wt = torch.rand_like(ix.weights)
    ix.weights.copy_(wt)
    ix.evict_into(dst, 20, 9)
    for l in range(2):
        for g in (0, 7):
            pos = R.kept_rows(wt[l, g].cpu().numpy(), st.rows, 20, 9)
            assert np.array_equal(host(dst.keys[l, g]).view(np.uint16), st.k[l][g, pos])
            assert np.array_equal(host(dst.values[l, g]).view(np.uint16), st.v[l][g, pos])


def test_long_own_text():
    """Own tokens by the thousands in front of few queries, and a whole long prompt."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(16)
    for heads, nq, text in (((8, 2, 64), 3, 9000), ((4, 1, 128), 1500, 0)):
        st = Stream(rng, heads, [(3, 20)])
        own = Own(rng, heads, text + nq, room=70)
        q = bf(rng, heads[0], nq, heads[2], scale=1.5)
        log("case", heads, nq, text)
        out, lse = P.HistoryAttention([st.ix], slopes=torch.full((heads[0],), 0.5, device="cuda"))(0, [dev(q)], own=[own.arg])
        check((out[0], lse[0]), want(st, 0, q, own, slopes=np.full(heads[0], 0.5)))


def test_many_listed_frames():
    """Lists longer than one sorting block, in any order, with repeats, padding and frames out of range."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(17)
    st = Stream(rng, (4, 2, 64), [(900, 3), (300, 5)])
    q = bf(rng, 4, 4, 64)
    att = P.HistoryAttention([st.ix], slopes=torch.full((4,), 0.01, device="cuda"))
    for n in (1, 2, 511, 512, 513, 3000, 4096):
        ids = rng.integers(-5, 1210, n)
        kinds = (rng.random(n) < 0.3).astype(np.int32)
        log("listed", n)
        out, lse = att(0, [dev(q)], frames=torch.from_numpy(ids[None]).cuda(), kinds=torch.from_numpy(kinds[None]).cuda())
        ref = want(st, 0, q, frames=[int(i) for i, k in zip(ids, kinds) if k == 0], slopes=np.full(4, np.float64(np.float32(0.01))))
        check((out[0], lse[0]), ref, n)


def test_window_and_compaction():
    """Frames that left the detailed window are not seen, before and after compaction
    (bit for bit the same), and weights and values move along."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(21)
    heads = (8, 2, 64)
    st = Stream(rng, heads, [(30, 24)], L=2, n_recent=4)
    q = bf(rng, 8, 7, 64)
    slopes = torch.full((8,), 0.05, device="cuda")
    cl = P.LongClusters(st.ix, 24, 30, 0.5)
    w0 = torch.rand_like(st.ix.weights)
    st.ix.weights.copy_(w0)
    whole = st.ix.budget_split(1 << 40)
    per = 24 * 2 * 2 * 2 * (2 * 64 + 4) + (2 * 64 + 2 * 2 * 64) * 4 + 4
    assert whole == 0 and st.ix.budget_split(20 * per) == 10 and st.ix.budget_split(20 * per - 1) == 11
    cl.absorb(11, 11)
    outs = []
    lists = torch.tensor([[3, 10, 11, 29, 15]], device="cuda")
    for step in range(2):
        for att, fr in ((P.HistoryAttention([st.ix]), None), (P.HistoryAttention([st.ix], slopes=slopes), None),
                        (P.HistoryAttention([st.ix]), lists)):
            out, lse = att(1, [dev(q)], frames=fr)
            check((out[0], lse[0]), want(st, 1, q, frames=None if fr is None else fr[0].tolist(), first=11,
                                         slopes=None if att.slopes is None else np.full(8, np.float32(0.05)).astype(float)))
            outs.append((out[0], lse[0]))
        if step == 0:
            st.ix.compact()
    for a, b in zip(outs[:3], outs[3:]):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(st.ix.weights, w0[:, :, 11 * 24:])
    assert np.array_equal(host(st.ix.values), np.stack(st.v)[:, :, 11 * 24:].view(np.int16))
    # and appends go on behind
    ks, vs = [bf(rng, 2, 24, 64) for _ in range(2)], [bf(rng, 2, 24, 64) for _ in range(2)]
    assert st.ix.append_kv([dev(x) for x in ks], [dev(x) for x in vs], 1, 24) == 30
    assert np.array_equal(host(st.ix.values[:, :, -24:]), np.stack(vs).view(np.int16))
    assert not st.ix.weights[:, :, -24:].any()


@pytest.mark.parametrize("gone", [1, 3, 15, 29, 30])
def test_compaction_moves_values_and_weights(gone):
    """Kept parts longer and shorter than the dropped one, also none at all."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(gone)
    st = Stream(rng, (8, 2, 128), [(30, 7)], L=2)
    w0 = torch.rand_like(st.ix.weights)
    st.ix.weights.copy_(w0)
    P.LongClusters(st.ix, 7, 30, 0.5).absorb(gone, gone)
    st.ix.compact()
    assert st.ix.n_rows == (30 - gone) * 7 and st.ix.window() == (gone, gone)
    assert torch.equal(st.ix.weights, w0[:, :, gone * 7:])
    assert np.array_equal(host(st.ix.values), np.stack(st.v)[:, :, gone * 7:].view(np.int16))
    assert np.array_equal(host(st.ix.keys), np.stack(st.k)[:, :, gone * 7:].view(np.int16))
    q = bf(rng, 8, 2, 128)
    out, lse = P.HistoryAttention([st.ix])(1, [dev(q)])
    check((out[0], lse[0]), want(st, 1, q, first=gone))


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128), (16, 1, 128), (3, 1, 64)], ids=str)
@pytest.mark.parametrize("nq,runs", [(1, [(1, 1)]), (1, [(50, 49)]), (3, [(9, 33), (5, 128)]), (40, [(20, 31)]),
                                     (150, [(3, 65)])], ids=str)
def test_accumulate(heads, nq, runs):
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], nq])
    st = Stream(rng, heads, runs, L=2)
    q = bf(rng, heads[0], nq, heads[2], scale=1.5)
    slopes = np.linspace(-0.02, 0.3, heads[0]).astype(np.float32)
    some = [0, len(st.rows) - 1, 0, -3]
    for layer, softcap, sl, frames, decay in ((1, 0.0, None, None, 1.0), (0, 4.0, None, None, 0.0),
                                              (1, 0.0, slopes, None, 0.25), (0, 20.0, slopes, some, 0.5),
                                              (1, 0.0, None, some, 1.0)):
        log("case", heads, nq, runs, layer, softcap, sl is not None, frames is not None, decay)
        att = P.HistoryAttention([st.ix], softcap, None if sl is None else torch.from_numpy(sl).cuda())
        fr = None if frames is None else torch.tensor([frames], device="cuda")
        _, lse = att(layer, [dev(q)], frames=fr)
        lse[0][0, 0] = float("-inf")                      # a query that saw nothing
        before = torch.rand(st.ix.weights.shape, device="cuda")
        st.ix.weights.copy_(before)
        att.accumulate(layer, [dev(q)], lse, frames=fr, decay=decay)
        got, b0 = st.ix.weights.double().cpu().numpy(), before.double().cpu().numpy()
        k, _, keep, age = st.seen(layer, frames)
        w, b = R.weights(R.f64(q), k, lse[0].cpu().numpy(), heads[0] // heads[1], softcap,
                         None if sl is None else sl.astype(np.float64), age)
        ref, tol = decay * b0[layer], 2 * R.U * b0[layer]
        ref[:, keep] += w
        tol[:, keep] += b + 2 * R.U * (w + b0[layer][:, keep])
        bad = np.abs(got[layer] - ref) > tol
        assert not bad.any(), (int(bad.sum()), float(np.abs(got[layer] - ref).max()))
        assert np.array_equal(got[1 - layer], b0[1 - layer])


def test_accumulate_ragged_batch():
    """Streams of a batch of 17 get their own sums; each sums to the heads' queries."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(31)
    sts = [Stream(rng, (8, 2, 64), [(1 + s, 1 + 9 * s)]) for s in range(17)]
    qs = [dev(bf(rng, 8, 1 + s % 4, 64)) for s in range(17)]
    att = P.HistoryAttention([s.ix for s in sts])
    _, lse = att(0, qs)
    att.accumulate(0, qs, lse, decay=0.0)
    for s, st in enumerate(sts):
        k, _, _, _ = st.seen(0)
        w, b = R.weights(R.f64(host(qs[s])), k, lse[s].cpu().numpy(), 4)
        got = st.ix.weights[0].double().cpu().numpy()
        assert (np.abs(got - w) <= b).all(), s
        assert np.allclose(got.sum(1), 4 * (1 + s % 4), rtol=1e-5)


@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128)], ids=str)
@pytest.mark.parametrize("runs,recent,keep", [([(1, 1)], 0, 1), ([(20, 49)], 3, 7), ([(4, 64), (3, 5), (6, 65)], 2, 16),
                                              ([(3, 700), (2, 513)], 1, 100), ([(5, 30)], 0, 30), ([(5, 30)], 9, 4),
                                              ([(1030, 3)], 2, 2)], ids=str)
def test_evict(heads, runs, recent, keep):
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], keep])
    st = Stream(rng, heads, runs, L=3, n_recent=recent)
    n, F = st.k[0].shape[1], len(st.rows)
    w = np.round(rng.random((3, heads[1], n)).astype(np.float32) ** 4, 2)       # ties, at 0 most of all
    w[rng.random(w.shape) < 0.05] = -0.0
    w[rng.random(w.shape) < 0.02] *= -1
    w[rng.random(w.shape) < 0.01] = np.inf
    st.ix.weights.copy_(torch.from_numpy(w))
    dst = P.ShallowIndex(3, *heads, F + 1, n + 5, n_recent=1)
    dst.attach_values()
    for hi in (max(0, F - recent), max(0, F - recent) // 2, 0, max(0, F - recent)):
        log("case", heads, runs, keep, hi)
        dst.arena.fill_(255)
        dst.value_arena.fill_(255)
        st.ix.evict_into(dst, hi, keep)
        rows = [min(r, keep) if f < hi else r for f, r in enumerate(st.rows)]
        assert dst.n_frames == F and dst.n_rows == sum(rows) and dst.window() == (0, 0)
        ex, src = dst.export(), st.ix.export()
        assert ex["frame_offsets"] == [0] + np.cumsum(rows).tolist()
        assert np.array_equal(ex["desc"].view(np.uint32), src["desc"].view(np.uint32))
        for l in range(3):
            for g in range(heads[1]):
                pos = R.kept_rows(w[l, g], st.rows, hi, keep)
                assert np.array_equal(ex["rows"][l, g], st.k[l][g, pos]), (l, g)
                assert np.array_equal(host(dst.values[l, g]).view(np.uint16), st.v[l][g, pos])
                assert np.array_equal(dst.weights[l, g].cpu().numpy(), w[l, g, pos])
                assert np.array_equal(ex["counts"][l, g], src["counts"][l, g, pos])
        assert dst.arena.view(torch.bfloat16).view(-1)[dst.keys.shape[2] * heads[2]:(n + 5) * heads[2]].isnan().all()
    assert np.array_equal(src["rows"], np.stack(st.k))                          # src is as it was


def test_evicted_index_serves():
    """Retrieval, attention, further appends and clusters on what eviction left equal
    those on an index that was given the kept rows."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(41)
    heads = (8, 2, 64)
    st = Stream(rng, heads, [(40, 24)], L=2, n_recent=4)
    w = rng.random((2, 2, 960)).astype(np.float32)
    w[:] = w[:1, :1]                                    # the same rows for every (layer, KV head)
    st.ix.weights.copy_(torch.from_numpy(w))
    cl = P.LongClusters(st.ix, 24, 40, 0.5)
    cl.absorb(6, 6)
    dst = P.ShallowIndex(2, *heads, 40, 900, n_recent=4)
    dst.attach_values()
    st.ix.evict_into(dst, 36, 8)
    assert dst.window() == (6, 6) and dst.n_frames == 40 and dst.n_rows == 30 * 8 + 4 * 24
    pos = R.kept_rows(w[0, 0, 6 * 24:], [24] * 34, 30, 8) + 6 * 24
    kk, vv = [k[:, pos] for k in st.k], [v[:, pos] for v in st.v]
    ref = P.ShallowIndex(2, *heads, 44, 900, n_recent=4)
    ref.attach_values()
    filler = [dev(bf(rng, 2, 6, 64)) for _ in range(2)]
    ref.append_kv(filler, filler, 6, 1)
    P.LongClusters(ref, 1, 8, 0.5).absorb(2, 2)          # ids line up; the rest of the filler leaves below
    ref2 = P.LongClusters(ref, 1, 8, 0.5)
    ref.append_kv([dev(k[:, :240]) for k in kk], [dev(v[:, :240]) for v in vv], 30, 8)
    ref.append_kv([dev(k[:, 240:]) for k in kk], [dev(v[:, 240:]) for v in vv], 4, 24)
    ref2.absorb(6, 4)
    ref.compact()
    qs = [dev(bf(rng, 8, 3, 64)) for _ in range(2)]
    for x in (dst, ref):
        more = [dev(W.bf16_bits(np.full((2, 5, 64), 0.25 * (l + 1), np.float32))) for l in range(2)]
        x.append_kv(more, more, 1, 5)
    a = P.HistoryAttention([dst])(1, [qs[1]])
    b = P.HistoryAttention([ref])(1, [qs[1]])
    assert torch.equal(a[0][0], b[0][0]) and torch.equal(a[1][0], b[1][0])
    da, db = (P.Retriever([x], 16, 4).debug([qs]) for x in (dst, ref))
    assert np.array_equal(da["topk_pos"], db["topk_pos"]) and np.array_equal(da["vote_hist"][:, :35], db["vote_hist"][:, :35])
    assert np.array_equal(da["topk_score"].view(np.uint32), db["topk_score"].view(np.uint32))


def test_evict_capacity():
    import paper_2609_02780_amd as P
    st = Stream(np.random.default_rng(3), (4, 2, 64), [(10, 20)])
    for frames, rows in ((9, 200), (10, 79)):
        dst = P.ShallowIndex(1, 4, 2, 64, frames, rows)
        dst.attach_values()
        with pytest.raises(P.SSError) as e:
            st.ix.evict_into(dst, 10, 8)
        assert e.value.status == 3 and dst.info() == (0, 0)


def test_streams_and_graphs():
    """A call on another stream, and calls captured into two graphs and replayed between
    eager calls with new inputs, equal the eager ones bit for bit."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(51)
    heads = (8, 2, 64)
    st = Stream(rng, heads, [(200, 31)])
    own = Own(rng, heads, 40)
    par = torch.tensor([i - 1 if i % 5 else -1 for i in range(12)], dtype=torch.int32, device="cuda")
    lists = torch.tensor([[3, 7, 150]], device="cuda")
    att = P.HistoryAttention([st.ix], 20.0, torch.full((8,), 0.01, device="cuda"))
    q1, q2 = dev(bf(rng, 8, 12, 64)), dev(bf(rng, 8, 1, 64))

    def tree():
        return att(0, [q1], own=[own.arg], tree=[par])

    def evidence():
        out, lse = att(0, [q2], frames=lists)
        att.accumulate(0, [q2], lse, frames=lists, decay=0.0)
        return out, lse

    side = torch.cuda.Stream()
    for f in (tree, evidence):
        a = f()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            b = f()
        side.synchronize()
        assert torch.equal(a[0][0], b[0][0]) and torch.equal(a[1][0], b[1][0])
    c = att(0, [q1], own=[own.arg], tree=[par], stream=side)
    side.synchronize()
    d = tree()
    assert torch.equal(c[0][0], d[0][0])
    graphs = []
    for f in (tree, evidence):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = f()
        graphs.append((g, r, f))
    for rep in range(3):
        q1.copy_(dev(bf(rng, 8, 12, 64)))
        q2.copy_(dev(bf(rng, 8, 1, 64)))
        lists.copy_(torch.tensor([[rep, 199 - rep, 60]], device="cuda"))
        wants = []
        for g, r, f in graphs:
            e = f()
            wants.append((e[0][0].clone(), e[1][0].clone(), st.ix.weights.clone()))
        st.ix.weights.fill_(7.0)
        torch.cuda.synchronize()
        for g, r, f in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (g, r, f), e in zip(graphs, wants):
            assert torch.equal(r[0][0], e[0]) and torch.equal(r[1][0], e[1]), rep
        assert torch.equal(st.ix.weights, wants[1][2]), rep


def test_two_calls_at_once():
    """Calls that run at the same time on two streams, and two graphs replayed together,
    share nothing."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(55)
    st = Stream(rng, (28, 4, 128), [(300, 49)])
    att = P.HistoryAttention([st.ix], slopes=torch.full((28,), 0.01, device="cuda"))
    qs = [dev(bf(rng, 28, n, 128)) for n in (1, 40)]
    wants = [att(0, [q]) for q in qs]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(5):
        got = []
        for side, q in zip(sides, qs):
            with torch.cuda.stream(side):
                got.append([att(0, [q]) for _ in range(4)])
        torch.cuda.synchronize()
        for g, w in zip(got, wants):
            for x in g:
                assert torch.equal(x[0][0], w[0][0]) and torch.equal(x[1][0], w[1][0]), rep
    graphs = []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = att(0, [q])
        graphs.append((g, r))
    for rep in range(4):
        for side, (g, r) in zip(sides, graphs):
            with torch.cuda.stream(side):
                g.replay()
        torch.cuda.synchronize()
        for (g, r), w in zip(graphs, wants):
            assert torch.equal(r[0][0], w[0][0]) and torch.equal(r[1][0], w[1][0]), rep
            r[0][0].zero_()


def test_longest_prompt():
    """4,096 queries, the most of a call, each seeing another number of own tokens."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(56)
    heads = (2, 1, 64)
    st = Stream(rng, heads, [(2, 9)])
    own, q = Own(rng, heads, 4096), bf(rng, 2, 4096, 64, scale=1.5)
    out, lse = P.HistoryAttention([st.ix])(0, [dev(q)], own=[own.arg])
    check((out[0], lse[0]), want(st, 0, q, own))


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("heads,nq", [((8, 2, 128), 30), ((8, 2, 128), 75), ((16, 8, 64), 60), ((8, 2, 64), 75)], ids=str)
def test_many_columns_over_many_tiles(heads, nq, mixed):
    """120 and 300 query rows a KV head, each item with more than 1,024 / d tiles of 64 keys: 16
    streams share the card, so the 70 tiles are cut into 8 parts at most where d = 128, 4 where d = 64."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], heads[2], nq, mixed])
    st = Stream(rng, heads, [(30, 65), (41, 62)] if mixed else [(70, 64)])
    S = 16
    qs = [bf(rng, heads[0], nq, heads[2], scale=1.5) for _ in range(S)]
    owns = [Own(rng, heads, nq + 9 * s) for s in range(S)]
    slopes = np.linspace(-0.01, 0.2, heads[0]).astype(np.float32)
    par = np.array([rng.integers(-1, i) if i else -1 for i in range(nq)], dtype=np.int32)
    listed = [f for f in range(len(st.rows)) if f % 9 != 4] + [3, 3, -1, 400]
    listed = (listed + [-1] * 71)[:71]
    for what, softcap, sl, frames, tree in (("plain", 0.0, None, None, None), ("cap", 6.0, None, None, None),
                                            ("bias", 0.0, slopes, None, None), ("all", 30.0, slopes, listed, None),
                                            ("tree", 0.0, slopes, None, par)):
        log("case", heads, nq, mixed, what)
        att = P.HistoryAttention([st.ix] * S, softcap, None if sl is None else torch.from_numpy(sl).cuda())
        fr = None if frames is None else torch.tensor([frames] * S, device="cuda")
        out, lse = att(0, [dev(q) for q in qs], own=[o.arg for o in owns], frames=fr,
                       tree=None if tree is None else [torch.from_numpy(tree).cuda()] * S)
        for s in (0, 9, 15):
            check((out[s], lse[s]), want(st, 0, qs[s], owns[s], tree, frames, 0, softcap,
                                         None if sl is None else sl.astype(np.float64)), (what, s))


def test_closed_index():
    import paper_2609_02780_amd as P
    st = Stream(np.random.default_rng(57), (4, 2, 64), [(2, 8)])
    att = P.HistoryAttention([st.ix])
    st.ix.close()
    with pytest.raises(RuntimeError):
        att(0, [dev(bf(np.random.default_rng(1), 4, 1, 64))])


def random_call(seed):
    """A batch of streams of random shape and state, a random call on it, its weights and an
    eviction, all against the 64-bit forms."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([seed, 99])
    pick = lambda *x: x[int(rng.integers(len(x)))]
    heads = pick((4, 2, 64), (28, 4, 128), (16, 1, 64), (3, 1, 128), (8, 8, 64), (10, 2, 128))
    L, S = int(rng.integers(1, 4)), pick(1, 1, 2, 3, 5)
    layer = int(rng.integers(L))
    sts, firsts = [], []
    for s in range(S):
        runs = [(int(rng.integers(1, 30)), int(pick(1, 7, 16, 33, 50, 128, 200))) for _ in range(pick(1, 1, 2, 3))]
        st = Stream(rng, heads, runs, L=L, n_recent=int(rng.integers(0, 4)))
        first = 0
        if len(runs) == 1 and len(st.rows) > 4 and rng.random() < 0.4:      # some frames left, perhaps the arena too
            first = int(rng.integers(1, len(st.rows) - 3))
            P.LongClusters(st.ix, runs[0][1], 40, 0.3).absorb(first, first)
            if rng.random() < 0.5:
                st.ix.compact()
        sts.append(st)
        firsts.append(first)
    nqs = [int(pick(1, 1, 2, 5, 9, 20, 33, 70, 140)) for _ in range(S)]
    qs = [bf(rng, heads[0], n, heads[2], scale=float(pick(0.3, 1.5, 4.0))) for n in nqs]
    cap = float(pick(0.0, 0.0, 2.0, 15.0, 50.0))
    slopes = (rng.random(heads[0]) * 0.5 - 0.1).astype(np.float32) if rng.random() < 0.5 else None
    owns = [Own(rng, heads, n + int(pick(0, 1, 40, 200)), room=int(rng.integers(0, 9))) if rng.random() < 0.6 else None
            for n in nqs]
    pars = [np.array([int(rng.integers(-2, n + 2)) for _ in range(n)], np.int32) if o is not None and rng.random() < 0.4
            else None for n, o in zip(nqs, owns)]
    lists = kinds = None
    if rng.random() < 0.5:
        m = int(pick(1, 3, 20, 70))
        lists = rng.integers(-2, 60, (S, m))
        kinds = (rng.random((S, m)) < 0.2).astype(np.int32) if rng.random() < 0.5 else np.zeros((S, m), np.int32)
    log("seed", seed, heads, L, [x.rows[:1] + [len(x.rows)] for x in sts], firsts, nqs, cap, slopes is not None,
        [o and o.n for o in owns], [p is not None for p in pars], None if lists is None else lists.shape)
    att = P.HistoryAttention([x.ix for x in sts], cap, None if slopes is None else torch.from_numpy(slopes).cuda())
    kw = {} if lists is None else {"frames": torch.from_numpy(lists).cuda(), "kinds": torch.from_numpy(kinds).cuda()}
    qd = [dev(q) for q in qs]
    out, lse = att(layer, qd, own=[o and o.arg for o in owns],
                   tree=[None if p is None else torch.from_numpy(p).cuda() for p in pars], **kw)
    s64 = None if slopes is None else slopes.astype(np.float64)
    seen = [None if lists is None else [int(f) for f, k in zip(lists[s], kinds[s]) if k == 0] for s in range(S)]
    for s in range(S):
        check((out[s], lse[s]), want(sts[s], layer, qs[s], owns[s], pars[s], seen[s], firsts[s], cap, s64), s)
    before = []
    for x in sts:
        w = torch.rand(x.ix.weights.shape, device="cuda")
        x.ix.weights.copy_(w)
        before.append(w.double().cpu().numpy())
    decay = float(pick(0.0, 0.5, 1.0))
    att.accumulate(layer, qd, lse, decay=decay, **kw)
    for s, x in enumerate(sts):
        k, _, keep, age = x.seen(layer, seen[s], firsts[s])
        w, b = R.weights(R.f64(qs[s]), k, lse[s].cpu().numpy(), heads[0] // heads[1], cap, s64, age)
        got, b0 = x.ix.weights.double().cpu().numpy(), before[s]
        gone = len(x.frame) - got.shape[-1]                  # rows that compaction dropped
        live = (x.frame >= firsts[s])[gone:]
        ref = np.where(live, decay * b0[layer], b0[layer])
        tol = 2 * R.U * b0[layer]
        keep = keep[gone:]
        ref[:, keep] += w
        tol[:, keep] += b + 2 * R.U * (w + b0[layer][:, keep])
        assert (np.abs(got[layer] - ref) <= tol).all(), ("weights", s)
        others = [l for l in range(L) if l != layer]
        assert np.array_equal(got[others], b0[others])
    x, first = sts[0], firsts[0]
    hi = int(rng.integers(first, max(first, len(x.rows) - x.ix.desc.n_recent) + 1))
    keep_rows = int(pick(1, 3, 20, 64, 300))
    dst = P.ShallowIndex(L, *heads, len(x.rows), len(x.frame))
    dst.attach_values()
    x.ix.evict_into(dst, hi, keep_rows)
    w = x.ix.weights.cpu().numpy()
    tail = x.rows[first:]
    start = sum(x.rows[:first]) - (len(x.frame) - w.shape[-1])
    for l in range(L):
        for g in range(heads[1]):
            pos = R.kept_rows(w[l, g, start:], tail, hi - first, keep_rows)
            assert np.array_equal(dst.weights[l, g].cpu().numpy(), w[l, g, start:][pos])
            assert np.array_equal(host(dst.keys[l, g]).view(np.uint16), x.k[l][g, sum(x.rows[:first]):][pos])
            assert np.array_equal(host(dst.values[l, g]).view(np.uint16), x.v[l][g, sum(x.rows[:first]):][pos])


@pytest.mark.parametrize("seed", range(40))
def test_random_calls(seed):
    random_call(seed)


def test_together():
    """A question on a stream, as it is served: append, retrieve, assemble the evidence,
    attend over the history and over the evidence, note the weights, evict, and draft
    an answer over the thinned history."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(61)
    cfg = W.Config("together", 2, 8, 2, 64, 20, 6, 16, 4, n_frames=60, n_planted=3)
    spec = W.stream_specs(cfg)[0]
    qs, keys = W.make_stream(cfg, spec, seed=3)
    vals = [bf(rng, 2, 1200, 64) for _ in range(2)]
    st = Stream(rng, (8, 2, 64), [], L=2)
    st.ix = P.ShallowIndex(2, 8, 2, 64, 60, 1200, n_recent=5)
    st.ix.attach_values()
    st.ix.append_kv([dev(k) for k in keys], [dev(v) for v in vals], 60, 20)
    st.rows, st.k, st.v = [20] * 60, list(keys), vals
    qd = [dev(q) for q in qs]
    ids, _, _, _ = P.Retriever([st.ix], cfg.top_k, cfg.n_select)([qd])
    units, kinds, n = P.assemble_evidence([st.ix], ids, 5)
    att = P.HistoryAttention([st.ix], 30.0)
    for l in range(2):
        own = Own(rng, (8, 2, 64), 6)
        out, lse = att(l, [qd[l]], own=[own.arg])
        check((out[0], lse[0]), want(st, l, qs[l], own, softcap=30.0), "history")
        ev, elog = att(l, [qd[l]], own=[own.arg], frames=units, kinds=kinds)
        listed = [int(u) for u in units[0].cpu() if u >= 0]
        assert len(listed) == int(n[0])
        check((ev[0], elog[0]), want(st, l, qs[l], own, None, listed, softcap=30.0), "evidence")
        att.accumulate(l, [qd[l]], lse)
    w = st.ix.weights.cpu().numpy()
    assert (w > 0).all() and (w.sum(-1) < 4 * 6).all()      # the own tokens took the rest
    dst = P.ShallowIndex(2, 8, 2, 64, 60, 1200, n_recent=5)
    dst.attach_values()
    st.ix.evict_into(dst, 55, 6)
    thin = Stream(rng, (8, 2, 64), [], L=2)
    thin.ix, thin.rows = dst, [6] * 55 + [20] * 5
    pos = [[R.kept_rows(w[l, g], st.rows, 55, 6) for g in range(2)] for l in range(2)]
    thin.k = [np.stack([st.k[l][g, pos[l][g]] for g in range(2)]) for l in range(2)]
    thin.v = [np.stack([st.v[l][g, pos[l][g]] for g in range(2)]) for l in range(2)]
    draft = bf(rng, 8, 9, 64)
    own = Own(rng, (8, 2, 64), 6 + 9)
    par = np.array([-1, 0, 0, 1, 1, 2, -1, 6, 3], dtype=np.int32)
    out, lse = P.HistoryAttention([dst])(1, [dev(draft)], own=[own.arg], tree=[torch.from_numpy(par).cuda()])
    check((out[0], lse[0]), want(thin, 1, draft, own, par), "drafts")


def test_binding_refusals():
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(71)
    heads = (4, 2, 64)
    st = Stream(rng, heads, [(4, 8)])
    plain = P.ShallowIndex(1, 4, 2, 64, 4, 32)
    q, own = dev(bf(rng, 4, 3, 64)), Own(rng, heads, 5)
    att = P.HistoryAttention([st.ix])
    bad = [lambda: P.HistoryAttention([]), lambda: P.HistoryAttention([st.ix], slopes=torch.zeros(3, device="cuda")),
           lambda: P.HistoryAttention([st.ix], slopes=torch.zeros(4)), lambda: plain.values, lambda: plain.weights,
           lambda: att(0, []), lambda: att(0, [q.float()]), lambda: att(0, [q[:, :, :32]]), lambda: att(0, [q.cpu()]),
           lambda: att(0, [q.transpose(0, 1)]), lambda: att(0, [q], own=[]), lambda: att(0, [q], tree=[None]),
           lambda: att(0, [q], own=[(own.arg[0], own.arg[1][:, :4], 5)]),
           lambda: att(0, [q], own=[own.arg], tree=[torch.zeros(2, dtype=torch.int32, device="cuda")]),
           lambda: att(0, [q], own=[own.arg], tree=[torch.zeros(3, device="cuda")]),
           lambda: att(0, [q], kinds=torch.zeros((1, 2), dtype=torch.int32, device="cuda")),
           lambda: att(0, [q], frames=torch.zeros((2, 2), dtype=torch.int64, device="cuda")),
           lambda: att(0, [q], frames=torch.zeros((1, 2), dtype=torch.int32, device="cuda")),
           lambda: att(0, [q], frames=torch.zeros((1, 2), dtype=torch.int64)),
           lambda: att.accumulate(0, [q], []), lambda: att.accumulate(0, [q], [torch.zeros(4, 2, device="cuda")]),
           lambda: att.accumulate(0, [q], [torch.zeros(4, 3)]),
           lambda: st.ix.append_kv([q], [], 1, 3)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    for f in (lambda: att(1, [q]), lambda: att(0, [q], own=[(own.arg[0], own.arg[1], 2)]),
              lambda: att(0, [q], frames=torch.zeros((1, 0), dtype=torch.int64, device="cuda")),
              lambda: P.HistoryAttention([plain])(0, [q]), lambda: P.HistoryAttention([st.ix], -1.0)(0, [q]),
              lambda: att.accumulate(0, [q], [torch.zeros(4, 3, device="cuda")], decay=2.0),
              lambda: st.ix.append([q], 1, 3), lambda: st.ix.evict_into(st.ix, 4, 2),
              lambda: st.ix.attach_values()):
        with pytest.raises((P.SSError, ValueError)):
            f()
    torch.cuda.synchronize()
