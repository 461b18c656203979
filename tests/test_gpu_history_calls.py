"""Calls of attention, weights and eviction at once, on other streams and beyond one
pass or one launch, against serial calls and the 64-bit forms."""
import ctypes as C

import numpy as np
import pytest

import history_ref as R
from test_gpu_history_attention import Stream, bf, check, dev, log, want

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_02780_amd  # noqa: F401  (fails loudly without the built library)


@pytest.mark.parametrize("heads,nq,rows", [((16, 1, 128), 8, 32), ((16, 1, 128), 16, 16), ((3, 1, 64), 43, 16),
                                           ((4, 2, 64), 64, 1)], ids=str)
def test_small_accumulations_at_once(heads, nq, rows):
    """Weights of two layers, whose few partial sums would fit the least workspace, from two
    streams and from two graphs replayed together."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], nq, rows])
    st = Stream(rng, heads, [(1, rows)], L=2)
    att = P.HistoryAttention([st.ix])
    lib, nqs = P.lib(), (C.c_int32 * 1)(nq)
    prm = att._params(0, None, None)
    need = lib.ss_attend_accumulate_workspace_bytes(att._handles, 1, nqs, C.byref(prm))
    assert need > 256                                    # 256: a call that writes none
    assert att._workspace(need).data_ptr() != att._least.data_ptr()
    qs = [dev(bf(rng, heads[0], nq, heads[2], scale=1.5)) for _ in range(2)]
    lses = [att(l, [qs[l]])[1] for l in range(2)]
    for l in range(2):
        att.accumulate(l, [qs[l]], lses[l], decay=0.0)
    want = st.ix.weights.clone()
    for l in range(2):
        w, b = R.weights(R.f64(qs[l].view(torch.int16).cpu().numpy()), R.f64(st.k[l]), lses[l][0].cpu().numpy(),
                         heads[0] // heads[1])
        assert (np.abs(want[l].double().cpu().numpy() - w) <= b).all(), l
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for rep in range(4):
        st.ix.weights.fill_(7.0)
        torch.cuda.synchronize()
        for l, side in enumerate(sides):
            with torch.cuda.stream(side):
                for _ in range(6):
                    att.accumulate(l, [qs[l]], lses[l], decay=0.0)
        torch.cuda.synchronize()
        assert torch.equal(st.ix.weights, want), rep
    graphs = []
    for l in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(4):
                att.accumulate(l, [qs[l]], lses[l], decay=0.0)
        graphs.append(g)
    for rep in range(4):
        st.ix.weights.fill_(7.0)
        torch.cuda.synchronize()
        for side, g in zip(sides, graphs):
            with torch.cuda.stream(side):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(st.ix.weights, want), rep


@pytest.mark.parametrize("runs", [[(600, 3)], [(300, 3), (300, 2)]], ids=str)
def test_evict_in_several_launches(runs):
    """307,200 (frame, layer, KV head) items, where a launch takes 262,144."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(len(runs))
    st = Stream(rng, (16, 16, 64), runs, L=32)
    n = len(st.frame)
    w = np.round(rng.random((32, 16, n)).astype(np.float32), 1)
    st.ix.weights.copy_(torch.from_numpy(w))
    dst = P.ShallowIndex(32, 16, 16, 64, 600, n)
    dst.attach_values()
    dst.arena.fill_(255)
    dst.value_arena.fill_(255)
    st.ix.evict_into(dst, 590, 2)
    rows = [min(r, 2) if f < 590 else r for f, r in enumerate(st.rows)]
    assert dst.export()["frame_offsets"] == [0] + np.cumsum(rows).tolist()
    keys, values, weights = (x.view(torch.int16).cpu().numpy().view(np.uint16) for x in (dst.keys, dst.values, dst.weights))
    for l in range(32):
        for g in range(16):
            pos = R.kept_rows(w[l, g], st.rows, 590, 2)
            assert np.array_equal(keys[l, g], st.k[l][g, pos]), (l, g)
            assert np.array_equal(values[l, g], st.v[l][g, pos]), (l, g)
            assert np.array_equal(np.ascontiguousarray(weights[l, g]).view(np.float32), w[l, g, pos]), (l, g)


def test_arenas_are_kept_for_a_callers_stream(monkeypatch):
    """Every call that is given a stream tells torch's allocator that the stream uses the arenas,
    so that an index dropped right after the call keeps its memory until the work is done."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(81)
    heads = (8, 2, 64)
    src, dst = (Stream(rng, heads, [(6, 8)], extra=8).ix for _ in range(2))
    plain = P.ShallowIndex(1, *heads, 9, 72)
    cl = P.LongClusters(src, 8, 4, 0.5)
    q = dev(bf(rng, 8, 5, 64))
    k, v = dev(bf(rng, 2, 8, 64)), dev(bf(rng, 2, 8, 64))
    att, ret, ranker = P.HistoryAttention([src]), P.Retriever([src], 8, 2), P.PooledRanker([src], 2)
    lse, ids = att(0, [q])[1], ret([[q]])[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    record, used = torch.Tensor.record_stream, set()

    def note(t, stream):
        if stream == side:
            used.add(t.data_ptr())
        return record(t, stream)

    monkeypatch.setattr(torch.Tensor, "record_stream", note)
    both = lambda x: {x.arena.data_ptr(), x.value_arena.data_ptr()}
    cases = {
        "attention": (lambda: att(0, [q], stream=side), both(src)),
        "weights": (lambda: att.accumulate(0, [q], lse, stream=side), both(src)),
        "evict": (lambda: src.evict_into(dst, 6, 3, stream=side), both(src) | both(dst)),
        "append_kv": (lambda: src.append_kv([k], [v], 1, 8, stream=side), both(src)),
        "append": (lambda: plain.append([k], 1, 8, stream=side), {plain.arena.data_ptr()}),
        "retrieve": (lambda: ret([[q]], stream=side), both(src) | {ids.data_ptr()}),
        "noalloc": (lambda: ret.noalloc([[q]], stream=side), both(src) | {ids.data_ptr()}),
        "pooled": (lambda: ranker([[q]], stream=side), both(src)),
        "scores": (lambda: src.debug_scores([q], 0, 0, stream=side), both(src)),
        "absorb": (lambda: cl.absorb(2, 2, stream=side), both(src) | {cl.arena.data_ptr()}),
        "clusters": (lambda: cl.retrieve([q], 2, stream=side), both(src) | {cl.arena.data_ptr()}),
        "evidence": (lambda: P.assemble_evidence([src], ids, 1, clusters=[cl], stream=side,
                                                 cluster_ids=torch.zeros((1, 1), dtype=torch.int64, device="cuda")),
                     {cl.arena.data_ptr()}),
        "compact": (lambda: src.compact(stream=side), both(src)),
    }
    for name, (call, arenas) in cases.items():
        log("call", name)
        used.clear()
        call()
        assert arenas <= used, name
    torch.cuda.synchronize()


def test_buffers_come_from_the_callers_stream(monkeypatch):
    """What a call on a given stream fills is memory of that stream: memory of the current
    one may still be read by work whose owner has let go of it."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(82)
    heads = (8, 2, 64)
    st = Stream(rng, heads, [(6, 8)])
    cl = P.LongClusters(st.ix, 8, 4, 0.5)
    cl.absorb(1, 1)
    q = dev(bf(rng, 8, 70, 64))
    att = P.HistoryAttention([st.ix])
    two = P.HistoryAttention([st.ix, st.ix])
    listed = torch.tensor([[1, 3]], device="cuda")
    lse = att(0, [q])[1]
    cl.retrieve([q], 2)                                  # its kept workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    empty, record, made, read = torch.empty, torch.Tensor.record_stream, [], set()
    here = torch.cuda.current_stream()

    def note_empty(*a, **kw):
        made.append(torch.cuda.current_stream() == side)
        return empty(*a, **kw)

    def note_read(t, stream):
        if stream == here:
            read.add(t.data_ptr())
        return record(t, stream)

    monkeypatch.setattr(torch, "empty", note_empty)
    monkeypatch.setattr(torch.Tensor, "record_stream", note_read)
    cases = {
        "attention": lambda: (lambda r: [*r[0], *r[1]])(att(0, [q], frames=listed, stream=side)),
        "two streams": lambda: (lambda r: [*r[0], *r[1]])(two(0, [q, q], stream=side)),
        "weights": lambda: att.accumulate(0, [q], lse, frames=listed, stream=side) or [],
        "scores": lambda: [st.ix.debug_scores([q], 0, 0, stream=side)],
        "clusters": lambda: cl.retrieve([q], 2, stream=side),
        "evidence": lambda: P.assemble_evidence([st.ix], listed, 1, stream=side),
    }
    for name, call in cases.items():
        log("call", name)
        made.clear()
        read.clear()
        out = call()
        assert made and all(made), name
        assert {t.data_ptr() for t in out} <= read, name
    torch.cuda.synchronize()


def test_another_current_device(monkeypatch):
    """Every entry point of the value cache refuses an index of another device than the current
    one, where its kernels would run, and tensors of another device than the index."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(83)
    src, dst = (Stream(rng, (8, 2, 64), [(6, 8)], extra=8).ix for _ in range(2))
    q, k = dev(bf(rng, 8, 5, 64)), dev(bf(rng, 2, 8, 64))
    att = P.HistoryAttention([src])
    lse = att(0, [q])[1]
    before = src.weights.clone()

    class Elsewhere(torch.Tensor):
        device = torch.device("cuda", 1)

    away = k.as_subclass(Elsewhere)
    for ks, vs in (([away], [k]), ([k], [away])):
        with pytest.raises(ValueError, match="lives on cuda:1"):
            src.append_kv(ks, vs, 1, 8)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: att(0, [q]), lambda: att.accumulate(0, [q], lse), lambda: src.evict_into(dst, 6, 3),
                 lambda: src.append_kv([k], [k], 1, 8)):
        with pytest.raises(ValueError, match="not the current device"):
            call()
    monkeypatch.undo()
    assert src.info() == dst.info() == (6, 48) and torch.equal(src.weights, before)


def test_evicted_into_a_larger_recent_window():
    """An eviction leaves an index whose recent window reaches before its first detailed frame:
    where the budget puts the border, absorption takes it, and frames leave once there are enough."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(84)
    heads = (8, 2, 64)
    st = Stream(rng, heads, [(12, 8)])
    P.LongClusters(st.ix, 8, 12, 0.5).absorb(8, 8)
    dst = P.ShallowIndex(1, *heads, 20, 160, n_recent=6)
    dst.attach_values()
    st.ix.evict_into(dst, 8, 8)
    assert dst.window() == (8, 8) and dst.info() == (12, 32)
    cl = P.LongClusters(dst, 8, 12, 0.5)
    assert dst.budget_split(0) == 8
    cl.absorb(8, 0)
    for f in (7, 9):
        with pytest.raises(P.SSError, match="outside 8..8"):
            cl.absorb(f, 1)
    q = bf(rng, 8, 5, 64)
    assert int(P.Retriever([dst], 8, 2)([[dev(q)]])[3][0]) == 0
    out, lse = P.HistoryAttention([dst])(0, [dev(q)])
    check((out[0], lse[0]), want(st, 0, q, first=8))
    k, v = bf(rng, 2, 32, 64), bf(rng, 2, 32, 64)
    assert dst.append_kv([dev(k)], [dev(v)], 4, 8) == 12
    assert dst.budget_split(0) == 10
    cl.absorb(10, 2)
    assert dst.window() == (8, 10)


@pytest.mark.parametrize("heads,nq,rows", [((16, 16, 64), 600, 300), ((16, 8, 128), 300, 800), ((32, 8, 128), 100, 900),
                                           ((16, 16, 64), 300, 1100)], ids=str)
def test_weights_of_many_query_rows_in_one_share(heads, nq, rows):
    """More than the 256 query rows of a KV head that are staged at a time: the next ones add to what
    the first left.  16 streams fill the card, so that the query rows are not shared out (then the
    call has no partial sums and asks for the least workspace)."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], nq, rows])
    G = heads[0] // heads[1]
    assert G * nq > 256
    runs = [(rows // 50, 50)]
    sts = [Stream(rng, heads, runs) for _ in range(16)]
    qs = [bf(rng, heads[0], nq, heads[2], scale=1.5) for _ in range(16)]
    qd = [dev(q) for q in qs]
    slopes = np.linspace(-0.02, 0.3, heads[0]).astype(np.float32)
    some = list(range(len(sts[0].rows) - 1))
    for softcap, sl, frames, decay in ((0.0, None, None, 0.0), (0.0, None, None, 1.0), (20.0, slopes, None, 0.5),
                                       (20.0, slopes, some, 0.25)):
        log("case", heads, nq, rows, softcap, sl is not None, frames is not None, decay)
        att = P.HistoryAttention([x.ix for x in sts], softcap, None if sl is None else torch.from_numpy(sl).cuda())
        fr = None if frames is None else torch.tensor([frames] * 16, device="cuda")
        prm = att._params(0, fr, None)
        if frames is None:
            assert P.lib().ss_attend_accumulate_workspace_bytes(att._handles, 16, (C.c_int32 * 16)(*[nq] * 16),
                                                                C.byref(prm)) == 256
        _, lse = att(0, qd, frames=fr)
        before = []
        for x in sts:
            x.ix.weights.copy_(torch.rand(x.ix.weights.shape, device="cuda"))
            before.append(x.ix.weights[0].double().cpu().numpy())
        att.accumulate(0, qd, lse, frames=fr, decay=decay)
        for s in (0, 7, 15):
            k, _, keep, age = sts[s].seen(0, frames)
            w, b = R.weights(R.f64(qs[s]), k, lse[s].cpu().numpy(), G, softcap,
                             None if sl is None else sl.astype(np.float64), age)
            ref, tol = decay * before[s], 2 * R.U * before[s]
            ref[:, keep] += w
            tol[:, keep] += b + 2 * R.U * (w + before[s][:, keep])
            got = sts[s].ix.weights[0].double().cpu().numpy()
            assert (np.abs(got - ref) <= tol).all(), (s, float(np.abs(got - ref).max()))


@pytest.mark.parametrize("heads", [(8, 2, 64), (4, 1, 128)], ids=str)
def test_rows_beyond_the_caches(heads):
    """More than 256 MB of keys that one block reads (and of keys and values), which are loaded past
    the caches: attention of few to 120 query rows a KV head, with and without a list, and weights.

    Tolerances are those of history_ref with fewer additions in a row: a lane adds at most the p of
    its 32 keys of a tile, then one sum a tile of at least 64 keys and one a share, so a chain has
    at most n / 64 + 64 additions however the n rows are shared out."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(heads[2])
    Hq, Hk, d = heads
    G, F, per = Hq // Hk, 3534, 300
    n = F * per
    assert n * Hk * d * 2 > 256 << 20

    def rows():          # magnitudes of 1/8 to 2
        x = rng.integers(0, 1 << 16, (Hk, n, d), dtype=np.uint16)
        return (x & 0x807F) | (((x >> 7) & 3) + 124 << 7)

    k, v = rows(), rows()
    ix = P.ShallowIndex(1, *heads, F, n)
    ix.attach_values()
    ix.append_kv([dev(k)], [dev(v)], F, per)
    every = torch.arange(F, device="cuda").flip(0)[None].contiguous()
    chain = (n / 64 + 64) * R.U
    kh, vh = R.f64(k), R.f64(v)
    att = P.HistoryAttention([ix])
    for nq in (1, 40 // G, 60 // G, 120 // G):
        q = bf(rng, Hq, nq, d, scale=5.0)            # scores of some 4, so that few rows take most of the weight
        log("case", heads, nq)
        runs = [att(0, [dev(q)]), att(0, [dev(q)], frames=every)]
        qh, w, bw = R.f64(q), np.zeros((Hk, n)), np.zeros((Hk, n))
        for h in range(Hq) if nq == 1 else (0, Hq - 1):
            s, err = R.scores(qh[h], kh[h // G], 0.0, None, None)
            m = s.max(1, keepdims=True)
            e = err.max(1) + 8 * R.U * np.abs(m[:, 0]) + 4 * R.U
            p = np.exp(s - m)
            z = p.sum(1)
            lse, rel = m[:, 0] + np.log(z), 2 * e + chain
            p /= z[:, None]
            out, mag = p @ vh[h // G], p @ np.abs(vh[h // G])
            for o, y in runs:
                g, gl = o[0][h].double().cpu().numpy(), y[0][h].double().cpu().numpy()
                assert (np.abs(g - out) <= (R.H + 2 * rel)[:, None] * mag + R.H * np.abs(out) * (1 + R.H)).all(), h
                assert (np.abs(gl - lse) <= rel + 8 * R.U * (np.abs(lse) + 1)).all(), h
            if nq == 1:
                zz = runs[0][1][0][h].double().cpu().numpy()[:, None]
                x = np.exp(s - zz)
                w[h // G] += x[0]
                bw[h // G] += (x * (2 * (err + 8 * R.U * (np.abs(s) + np.abs(zz))) + (G + 8) * R.U))[0] + 2.0 ** -126
        if nq == 1:
            for fr in (None, every):
                att.accumulate(0, [dev(q)], runs[0][1], frames=fr, decay=0.0)
                assert (np.abs(ix.weights[0].double().cpu().numpy() - w) <= bw).all()


@pytest.mark.parametrize("rows", [1, 2, 7, 16, 31, 32, 40])
@pytest.mark.parametrize("heads", [(4, 2, 64), (28, 4, 128)], ids=str)
def test_steep_bias(heads, rows):
    """Under a steep bias the newest frame takes all weight, and its score is as precise as a product
    of its own age: not rounded at the bias of the older frames that share its group of 32 keys.

    To first order an error e_j of q.k moves the log of the sum by sum_j p_j e_j, which is doubled
    here; its sum adds n + 64 roundings.  At the magnitude of the bias there are at most 7: of log2 e,
    of the slope in units of log 2, of the bias, of the biased score, of maximum + log2 of the sum, of
    ln 2 and of the product with it."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], rows])
    st = Stream(rng, heads, [(96, rows)])                # whole groups of 32 rows: their last row is the newest
    q = bf(rng, heads[0], 3, heads[2])
    k, v, _, age = st.seen(0)
    for slope in (0.7, 30.0, 300.0):
        slopes = np.full(heads[0], slope, np.float32)
        log("case", heads, rows, slope)
        out, lse = P.HistoryAttention([st.ix], slopes=torch.from_numpy(slopes).cuda())(0, [dev(q)])
        for h in range(heads[0]):
            s, err = R.scores(R.f64(q[h]), k[h // (heads[0] // heads[1])], 0.0, None, None)
            s = s - float(slopes[h]) * age
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            z = p.sum(1)
            ref = m[:, 0] + np.log(z)
            tol = 2 * (p * err).sum(1) / z + (len(age) + 64) * R.U + 7 * R.U * (np.abs(ref) + 1)
            got = lse[0][h].double().cpu().numpy()
            assert (np.abs(got - ref) <= tol).all(), (slope, h, float((np.abs(got - ref) / tol).max()))


@pytest.mark.parametrize("heads,nq", [((4, 2, 64), 1), ((28, 4, 128), 17), ((16, 1, 64), 60), ((8, 8, 128), 200)], ids=str)
def test_without_lse(heads, nq):
    """A C caller may leave the logs out: the outputs are the same."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng([heads[0], nq])
    st = Stream(rng, heads, [(21, 33)])
    q = dev(bf(rng, heads[0], nq, heads[2], scale=1.5))
    att = P.HistoryAttention([st.ix])
    expected = att(0, [q])[0][0]
    out, lib, nqs, prm = torch.full_like(expected, 5.0), P.lib(), (C.c_int32 * 1)(nq), att._params(0, None, None)
    need = lib.ss_attend_workspace_bytes(att._handles, 1, nqs, None, C.byref(prm))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert lib.ss_attend(att._handles, 1, (C.c_void_p * 1)(q.data_ptr()), nqs, None, C.byref(prm), ws.data_ptr(), need,
                         torch.cuda.current_stream().cuda_stream, (C.c_void_p * 1)(out.data_ptr()), None) == 0
    assert torch.equal(out, expected)


@pytest.mark.parametrize("nq", [2, 90])
def test_three_groups_of_streams_with_lists(nq):
    """33 streams with frames of two sizes, lists, cap and bias: attention and decayed weights."""
    import paper_2609_02780_amd as P
    rng = np.random.default_rng(nq)
    sts = [Stream(rng, (4, 2, 64), [(1 + s % 5, 1 + s), (2, 9)]) for s in range(33)]
    qs = [bf(rng, 4, nq + s % 3, 64, scale=1.5) for s in range(33)]
    qd, slopes = [dev(q) for q in qs], np.linspace(-0.05, 0.3, 4).astype(np.float32)
    lists = rng.integers(-1, 9, (33, 5))
    frames = torch.from_numpy(lists).cuda()
    att = P.HistoryAttention([x.ix for x in sts], 12.0, torch.from_numpy(slopes).cuda())
    out, lse = att(0, qd, frames=frames)
    for x in sts:
        x.ix.weights.fill_(2.0)
    att.accumulate(0, qd, lse, frames=frames, decay=0.5)
    for s, x in enumerate(sts):
        seen, s64 = lists[s].tolist(), slopes.astype(np.float64)
        check((out[s], lse[s]), want(x, 0, qs[s], None, None, seen, 0, 12.0, s64), s)
        k, _, keep, age = x.seen(0, seen)
        w, b = R.weights(R.f64(qs[s]), k, lse[s].cpu().numpy(), 2, 12.0, s64, age)
        ref = np.ones((2, len(keep)))
        tol = np.full_like(ref, 4 * R.U)
        ref[:, keep] += w
        tol[:, keep] += b + 2 * R.U * (w + 1)
        assert (np.abs(x.ix.weights[0].double().cpu().numpy() - ref) <= tol).all(), s
