"""Attention over a stream's stored history, and eviction by its weight: the
calls whose speed counts.

Four operators over an index that keeps values beside its keys.  For one layer,
query head h reads KV head h // G; rows are those of the detailed frames.

``attend``      out = sum_j p_j v_j,  p = softmax_j(s_j) over the visible rows and
                the question's own tokens (the last n_q of n_own are the queries,
                each sees the own tokens up to itself);
                s = cap(q.k / sqrt(d)) - slope_h * age,  cap(x) = c tanh(x / c) or
                x,  age = frames stored - the row's frame id (own tokens: 0).  A
                list of frames restricts the rows to those frames.  Also the
                natural log of the normaliser.
``tree``        the same where the queries are drafted tokens: each sees the text
                before the drafts, its ancestors and itself.
``accumulate``  w_j = decay w_j + sum over queries and the G heads of
                exp(s_j - lse), one number a stored row.
``evict``       every frame before a border keeps its ``keep`` rows of the largest
                weight for each (layer, KV head), in their order, ties to the
                earlier row; later frames stay whole.

``listed()`` gives the cases, ``draw(rng)`` one more of the same ranges.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------

def _attend(name, frames, tokens, heads, n_q, **kw):
    c = {"name": name, "op": "attend", "frames": frames, "frames_least": frames, "streams": 1, "tokens": tokens,
         "tokens_late": tokens, "q_heads": heads[0], "kv_heads": heads[1], "d": heads[2], "layers": 2, "layer": 1,
         "n_q": n_q, "text": 0, "own": False, "softcap": 0.0, "bias": False, "listed": 0}
    c.update(kw)
    return c


def listed():
    return [
        # one decoded token over a tiny index (64 frames of 16 tokens, 4/2 heads, d 64): latency
        _attend("attend_token_tiny", 64, 16, (4, 2, 64), 1),
        # one decoded token over the 1-hour stream, with a bias for each head on the frames' age
        _attend("attend_token_1h", 3600, 196, (28, 4, 128), 1, text=37, own=True, bias=True),
        # one decoded token for each of 8 streams of different length, capped scores
        _attend("attend_streams", 1800, 196, (16, 2, 128), 1, streams=8, frames_least=300, text=100, own=True,
                softcap=30.0),
        # a question of 64 tokens over the 1-hour stream (the shallow query forward)
        _attend("attend_question_1h", 3600, 196, (28, 4, 128), 64, own=True),
        # a prompt of 1,024 tokens over the 10-minute stream
        _attend("attend_prompt_10min", 600, 196, (28, 4, 128), 1024, own=True),
        # the question over the evidence frames alone: 32 selected, their neighbours, some twice
        _attend("attend_evidence", 3600, 196, (28, 4, 128), 64, own=True, listed=70, softcap=50.0),
        # 13 drafted tokens behind 200 of text, over 300 frames of 49 and 196 tokens, d 64
        _attend("tree_small", 300, 49, (16, 4, 64), 13, op="tree", tokens_late=196, text=200, own=True),
        # 64 drafted tokens behind 300 of text over the 1-hour stream
        _attend("tree_1h", 3600, 196, (28, 4, 128), 64, op="tree", text=300, own=True),
        # the weight that the last token gives each row of the 1-hour stream
        _attend("accumulate_token_1h", 3600, 196, (28, 4, 128), 1, op="accumulate"),
        # the weight that a question of 32 tokens gives each row of 10 minutes, capped scores and a bias
        _attend("accumulate_question", 600, 196, (28, 4, 128), 32, op="accumulate", softcap=30.0, bias=True),
        # eviction of a tiny index: 64 frames of 16 tokens to 4 rows, the newest 4 frames whole
        _evict("evict_tiny", 64, 16, (4, 2, 64), 2, 4, 4),
        # eviction of the 1-hour stream, 196 rows to 32 a frame, the newest 6 frames whole
        _evict("evict_1h", 3600, 196, (28, 4, 128), 4, 32, 6),
    ]


def _evict(name, frames, tokens, heads, layers, keep, recent):
    return {"name": name, "op": "evict", "frames": frames, "frames_least": frames, "streams": 1, "tokens": tokens,
            "tokens_late": tokens, "q_heads": heads[0], "kv_heads": heads[1], "d": heads[2], "layers": layers,
            "keep": keep, "recent": recent}


_HEADS = ((4, 2, 64), (16, 4, 64), (16, 2, 128), (28, 4, 128), (8, 8, 128), (16, 1, 128), (3, 1, 64))


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attend", "attend", "tree", "accumulate", "evict"))
    heads = rng.choice(_HEADS)
    frames = _log_int(rng, 1, 3600)
    tokens = rng.choice((rng.randint(1, 260), 196, _log_int(rng, 1, 800)))
    late = rng.choice((tokens, rng.randint(1, 260)))
    if op == "evict":
        c = _evict("", frames, tokens, heads, rng.randint(1, 4), _log_int(rng, 1, 256), rng.randint(0, 8))
        c["tokens_late"] = late
    else:
        n_q = _log_int(rng, 1, 256 if op == "tree" else 1024)
        own_ = op == "tree" or (op == "attend" and rng.random() < 0.7)
        c = _attend("", frames, tokens, heads, n_q, op=op, tokens_late=late, own=own_,
                    text=rng.choice((0, _log_int(rng, 1, 1000))) if own_ else 0,
                    softcap=rng.choice((0.0, 0.0, 20.0, 50.0)), bias=rng.random() < 0.4,
                    listed=_log_int(rng, 1, 100) if rng.random() < 0.3 else 0, layers=rng.randint(1, 3))
        c["layer"] = rng.randrange(c["layers"])
        if rng.random() < 0.3:
            c["streams"] = rng.randint(2, 8)
            c["frames_least"] = rng.randint(1, frames)
    del c["name"]
    top = [work(x) for x in listed()]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    while any(work(c)[k] > most[k] or _arena(c) > 6e9 for k in most):
        c["frames"] = max(1, c["frames"] * 2 // 3)
        c["frames_least"] = min(c["frames_least"], c["frames"])
    return c


def _lengths(case):
    """Frames of each stream."""
    S, lo, hi = case["streams"], case["frames_least"], case["frames"]
    return [hi if S == 1 else lo + (hi - lo) * ((s * 5) % S) // (S - 1) if S % 5 else lo + (hi - lo) * s // (S - 1)
            for s in range(S)]


def _frame_rows(case, frames):
    """Rows of each frame: the second half of a stream may come with another number of tokens."""
    half = frames // 2 if case["tokens_late"] != case["tokens"] else frames
    return [case["tokens"]] * half + [case["tokens_late"]] * (frames - half)


def _arena(case):
    return sum(sum(_frame_rows(case, f)) for f in _lengths(case)) * case["layers"] * case["kv_heads"] * case["d"] * 4


def _list_of(case, frames, s):
    """Listed frames of stream s, with repeats and padding among them, as numpy int64."""
    rng = np.random.default_rng([frames, case["listed"], s])
    ids = rng.integers(0, frames, case["listed"])
    if case["listed"] > 4:
        ids[1] = -1
        ids[3] = ids[0]
    return ids


def _visible_rows(case, s, frames):
    rows = _frame_rows(case, frames)
    if not case.get("listed"):
        return sum(rows)
    return sum(rows[f] for f in set(int(i) for i in _list_of(case, frames, s)) if f >= 0)


def work(case):
    Hq, Hk, d = case["q_heads"], case["kv_heads"], case["d"]
    if case["op"] == "evict":
        rows = _frame_rows(case, case["frames"])
        border = max(0, case["frames"] - case["recent"])
        thin = sum(min(case["keep"], r) for r in rows[:border])
        kept = thin + sum(rows[border:])
        per = case["layers"] * Hk
        # every weight read once, kept rows (key, value, member count, weight) read and written,
        # and each frame's descriptor and mean keys moved
        return {"bytes": per * (4 * sum(rows) + kept * (2 * (4 * d + 4) + 4))
                + case["frames"] * 8 * Hk * d * (1 + case["layers"]), "flops": 0}
    total_b = total_f = 0
    n_q = case["n_q"]
    for s, frames in enumerate(_lengths(case)):
        n = _visible_rows(case, s, frames)
        n_own = case["text"] + n_q if case["own"] else 0
        pairs = n_q * n + (n_q * case["text"] + n_q * (n_q + 1) // 2 if case["own"] else 0)
        if case["op"] == "accumulate":
            total_b += Hk * n * (2 * d + 4) + Hq * n_q * (2 * d + 4)
            total_f += 2 * Hq * d * pairs
        else:
            total_b += Hk * (n + n_own) * 4 * d + Hq * n_q * (4 * d + 4)
            total_f += 4 * Hq * d * pairs
    return {"bytes": total_b, "flops": total_f}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _bf16_normal(gen, *shape, scale=1.0):
    return torch.randn(*shape, generator=gen, device=_DEV, dtype=torch.bfloat16) * scale


def _rows_of(gen, case, frames, scale):
    """Rows [H_kv][N][d] of one layer: a centre for each frame and a spread around it."""
    rows = torch.tensor(_frame_rows(case, frames), device=_DEV)
    centre = _bf16_normal(gen, case["kv_heads"], frames, case["d"], scale=scale)
    n = int(rows.sum())
    x = _bf16_normal(gen, case["kv_heads"], n, case["d"], scale=0.5 * scale)
    return x + torch.repeat_interleave(centre, rows, dim=1, output_size=n)


def _parents(case, seed, s):
    """A drafted tree: each token's parent is an earlier draft or the text (-1)."""
    rng = np.random.default_rng([seed, s, 7])
    return np.array([-1 if i == 0 or rng.random() < 0.1 else rng.integers(max(0, i - 6), i)
                     for i in range(case["n_q"])], dtype=np.int32)


def _ancestors(parents):
    """[n][n] truth: j is i or an ancestor of i."""
    n = len(parents)
    m = np.eye(n, dtype=bool)
    for i in range(n):
        if parents[i] >= 0:
            m[i] |= m[parents[i]]
    return m


def _own_mask(case, seed, s):
    """[n_q][n_own] truth of the own tokens that each query sees."""
    n_q, text = case["n_q"], case["text"]
    tail = _ancestors(_parents(case, seed, s)) if case["op"] == "tree" else np.tril(np.ones((n_q, n_q), dtype=bool))
    return torch.from_numpy(np.concatenate([np.ones((n_q, text), dtype=bool), tail], 1)).to(_DEV)


def _slopes(case):
    """Slopes 2^(-8 (h + 1) / H_q) / 64 for each query head: the far end of an hour stays in reach."""
    h = torch.arange(1, case["q_heads"] + 1, dtype=torch.float64)
    return (torch.exp2(-8.0 * h / case["q_heads"]) / 64.0).float().to(_DEV)


def _inputs(case, seed):
    """Per stream, everything that the call is given; the same for every form."""
    out = []
    for s, frames in enumerate(_lengths(case)):
        gen = torch.Generator(device=_DEV)
        gen.manual_seed(seed * 1009 + s)
        x = {"frames": frames}
        x["keys"] = [_rows_of(gen, case, frames, 1.0) for _ in range(case["layers"])]
        x["values"] = [_rows_of(gen, case, frames, 1.0) for _ in range(case["layers"])]
        n = x["keys"][0].shape[1]
        if case["op"] == "evict":
            w = torch.rand((case["layers"], case["kv_heads"], n), generator=gen, device=_DEV)
            x["weights"] = torch.where(w < 0.2, torch.zeros_like(w), w ** 8)   # most weight on few rows, many ties at 0
            out.append(x)
            continue
        Hq, Hk, d, n_q = case["q_heads"], case["kv_heads"], case["d"], case["n_q"]
        x["q"] = _bf16_normal(gen, Hq, n_q, d, scale=1.5)
        if case["own"]:
            x["n_own"] = case["text"] + n_q
            cap = x["n_own"] + 5                  # a growing cache: room behind the last token
            x["own_k"] = _bf16_normal(gen, Hk, cap, d)
            x["own_v"] = _bf16_normal(gen, Hk, cap, d)
        if case["op"] == "accumulate":
            x["lse"] = _normaliser(case, x, s)
        out.append(x)
    return out


def _row_index(case, s, frames):
    """Positions of the visible rows (None: all) and each row's age in frames."""
    rows = torch.tensor(_frame_rows(case, frames), device=_DEV)
    frame = torch.repeat_interleave(torch.arange(frames, device=_DEV), rows)
    keep = None
    if case["listed"]:
        ids = torch.from_numpy(_list_of(case, frames, s)).to(_DEV)
        keep = torch.isin(frame, ids[ids >= 0]).nonzero().flatten()
        frame = frame[keep]
    return keep, frames - frame


def _normaliser(case, x, s):
    """The log of each query's sum over the visible rows, as the attention of the call before left it."""
    keep, age = _row_index(case, s, x["frames"])
    k = x["keys"][case["layer"]]
    k = (k if keep is None else k[:, keep]).double()
    G = case["q_heads"] // case["kv_heads"]
    sl = _slopes(case).double()
    out = torch.empty(case["q_heads"], case["n_q"], device=_DEV, dtype=torch.float32)
    for h in range(case["q_heads"]):
        z = torch.matmul(x["q"][h].double(), k[h // G].t()) / math.sqrt(case["d"])
        if case["softcap"]:
            z = case["softcap"] * torch.tanh(z / case["softcap"])
        if case["bias"]:
            z = z - sl[h] * age
        out[h] = torch.logsumexp(z, 1).float()
    return out


def prepare(case, seed):
    ins = _inputs(case, seed)
    st = {"case": case}
    if case["op"] == "tree":
        st["parents"] = [torch.from_numpy(_parents(case, seed, s)).to(_DEV) for s in range(case["streams"])]
    if not own:
        st["ins"] = ins
        if case["op"] != "evict":
            st["slopes"] = _slopes(case)
            st["lists"] = _device_lists(case, ins)
        return st
    import paper_2609_02780_amd as P
    st["index"] = []
    for x in ins:
        rows = _frame_rows(case, x["frames"])
        n = sum(rows)
        ix = P.ShallowIndex(case["layers"], case["q_heads"], case["kv_heads"], case["d"], x["frames"], n,
                            n_recent=case.get("recent", 0))
        ix.attach_values()
        half = rows.count(rows[0]) if rows[0] != rows[-1] else len(rows)
        ix.append_kv([k[:, :half * rows[0]].contiguous() for k in x["keys"]],
                     [v[:, :half * rows[0]].contiguous() for v in x["values"]], half, rows[0])
        if half < len(rows):
            ix.append_kv([k[:, half * rows[0]:].contiguous() for k in x["keys"]],
                         [v[:, half * rows[0]:].contiguous() for v in x["values"]], len(rows) - half, rows[-1])
        st["index"].append(ix)
        if case["op"] == "evict":
            ix.weights.copy_(x["weights"])
            st["thin"] = P.ShallowIndex(case["layers"], case["q_heads"], case["kv_heads"], case["d"], x["frames"], n,
                                        n_recent=case["recent"])
            st["thin"].attach_values()
    if case["op"] != "evict":
        st["attention"] = P.HistoryAttention(st["index"], softcap=case["softcap"],
                                             slopes=_slopes(case) if case["bias"] else None)
        st["q"] = [x["q"] for x in ins]
        st["lists"] = _device_lists(case, ins)
        if case["own"]:
            st["own"] = [(x["own_k"], x["own_v"], x["n_own"]) for x in ins]
        if case["op"] == "accumulate":
            st["lse"] = [x["lse"] for x in ins]
    return st


def _device_lists(case, ins):
    if not case["listed"]:
        return None
    return torch.from_numpy(np.stack([_list_of(case, x["frames"], s) for s, x in enumerate(ins)])).to(_DEV)


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["op"] == "evict":
        return _plain_evict(case, state["ins"][0])
    if case["op"] == "accumulate":
        return [_plain_accumulate(case, state, s) for s in range(case["streams"])]
    return [_plain_attend(case, state, s) for s in range(case["streams"])]


def _run_own(case, st):
    if case["op"] == "evict":
        ix, thin = st["index"][0], st["thin"]
        ix.evict_into(thin, max(0, case["frames"] - case["recent"]), case["keep"])
        return [thin.keys, thin.values, thin.weights]
    if case["op"] == "accumulate":
        st["attention"].accumulate(case["layer"], st["q"], st["lse"], frames=st["lists"], decay=0.0)
        return [ix.weights[case["layer"]] for ix in st["index"]]
    out, lse = st["attention"](case["layer"], st["q"], own=st.get("own"), tree=st.get("parents"), frames=st["lists"])
    return list(zip(out, lse))


def _plain_rows(case, state, s):
    """Visible keys and values in 32 bits, their positions, and the rows' age."""
    x = state["ins"][s]
    k, v = x["keys"][case["layer"]], x["values"][case["layer"]]
    rows = torch.tensor(_frame_rows(case, x["frames"]), device=k.device)
    keep, age = None, None
    if case["listed"] or case["bias"]:
        frame = torch.repeat_interleave(torch.arange(x["frames"], device=k.device), rows, output_size=k.shape[1])
        if case["listed"]:
            mark = torch.zeros(x["frames"] + 1, dtype=torch.bool, device=k.device)
            ids = state["lists"][s]
            mark[torch.where(ids < 0, x["frames"], ids)] = True
            keep = mark[frame].nonzero().flatten()
            frame, k, v = frame[keep], k[:, keep], v[:, keep]
        age = (x["frames"] - frame).float()
    return k, v, keep, age


def _plain_scores(case, state, q, k, age, h0, h1):
    """Scores of KV heads [h0, h1): [heads][G][n_q][rows] in 32 bits."""
    G = case["q_heads"] // case["kv_heads"]
    n_q = q.shape[1]
    qf = q[h0 * G:h1 * G].float().reshape(h1 - h0, G * n_q, case["d"])
    s = torch.matmul(qf, k[h0:h1].float().transpose(1, 2).contiguous()) * (1.0 / math.sqrt(case["d"]))
    if case["softcap"]:
        s = case["softcap"] * torch.tanh(s / case["softcap"])
    s = s.reshape(h1 - h0, G, n_q, -1)
    if case["bias"] and age is not None:
        s = s - state["slopes"][h0 * G:h1 * G].reshape(h1 - h0, G, 1, 1) * age
    return s


def _heads_at_once(case, n):
    G = case["q_heads"] // case["kv_heads"]
    return max(1, min(case["kv_heads"], (1 << 31) // max(1, G * case["n_q"] * n)))


def _plain_attend(case, state, s):
    x = state["ins"][s]
    q = x["q"]
    k, v, _, age = _plain_rows(case, state, s)
    n, n_q, n_own = k.shape[1], case["n_q"], 0
    mask = None
    if case["own"]:
        n_own = x["n_own"]
        k = torch.cat([k, x["own_k"][:, :n_own]], 1)
        v = torch.cat([v, x["own_v"][:, :n_own]], 1)
        if age is not None:
            age = torch.cat([age, age.new_zeros(n_own)])
        mask = torch.ones(n_q, n + n_own, dtype=torch.bool, device=q.device)
        if case["op"] == "tree":
            # i sees its parent; squaring the relation doubles its reach
            par = state["parents"][s].long()
            at = torch.arange(n_q, device=q.device)
            see = (at == at[:, None]) | (at == par[:, None])
            for _ in range(max(1, (n_q - 1).bit_length())):
                see = torch.matmul(see.float(), see.float()) > 0
        else:
            see = torch.ones(n_q, n_q, dtype=torch.bool, device=q.device).tril()
        mask[:, n + n_own - n_q:] = see
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    step = _heads_at_once(case, k.shape[1])
    G = case["q_heads"] // case["kv_heads"]
    for h0 in range(0, case["kv_heads"], step):
        h1 = min(case["kv_heads"], h0 + step)
        sc = _plain_scores(case, state, q, k, age, h0, h1)
        if mask is not None:
            sc = sc.masked_fill(~mask, float("-inf"))
        top = sc.amax(-1, keepdim=True)
        top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
        p = torch.exp(sc - top)
        z = p.sum(-1, keepdim=True)
        o = torch.matmul(p.reshape(h1 - h0, G * n_q, -1), v[h0:h1].float()).reshape(h1 - h0, G, n_q, -1)
        out[h0 * G:h1 * G] = torch.where(z > 0, o / z, torch.zeros_like(o)).reshape((h1 - h0) * G, n_q, -1).to(out.dtype)
        lse[h0 * G:h1 * G] = (top + torch.log(z)).reshape((h1 - h0) * G, n_q)
    return out, lse


def _plain_accumulate(case, state, s):
    x = state["ins"][s]
    k, _, keep, age = _plain_rows(case, state, s)
    w = torch.zeros(case["kv_heads"], x["keys"][0].shape[1], dtype=torch.float32, device=k.device)
    step = _heads_at_once(case, k.shape[1])
    G = case["q_heads"] // case["kv_heads"]
    for h0 in range(0, case["kv_heads"], step):
        h1 = min(case["kv_heads"], h0 + step)
        sc = _plain_scores(case, state, x["q"], k, age, h0, h1)
        p = torch.exp(sc - x["lse"][h0 * G:h1 * G].reshape(h1 - h0, G, case["n_q"], 1))
        t = p.sum((1, 2))
        if keep is None:
            w[h0:h1] = t
        else:
            w[h0:h1, keep] = t
    return w


def _plain_evict(case, x):
    """The rows that stay, gathered: keys, values and weights."""
    rows = _frame_rows(case, x["frames"])
    border = max(0, x["frames"] - case["recent"])
    w = x["weights"]
    parts, lo = [], 0
    f = 0
    while f < len(rows):
        g = f
        while g < len(rows) and rows[g] == rows[f] and (g < border) == (f < border):
            g += 1
        n, r = g - f, rows[f]
        base = lo + torch.arange(n, device=w.device)[:, None] * r
        if f < border and case["keep"] < r:
            sub = w[:, :, lo:lo + n * r].reshape(*w.shape[:2], n, r)
            best = torch.sort(sub, dim=-1, descending=True, stable=True)[1][..., :case["keep"]]
            pos = base + torch.sort(best, dim=-1)[0]
        else:
            pos = (base + torch.arange(r, device=w.device)).expand(*w.shape[:2], n, r)
        parts.append(pos.reshape(*w.shape[:2], -1))
        lo += n * r
        f = g
    pos = torch.cat(parts, -1)
    pick = pos[..., None].expand(*pos.shape, case["d"])
    return [torch.gather(torch.stack(x["keys"]), 2, pick), torch.gather(torch.stack(x["values"]), 2, pick),
            torch.gather(w, 2, pos)]


# --------------------------------------------------------------------------
# The definition in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    ins = _inputs(case, seed)
    if case["op"] == "evict":
        return _exact_evict(case, ins[0])
    res = []
    G = case["q_heads"] // case["kv_heads"]
    scale = 1.0 / math.sqrt(case["d"])
    sl = _slopes(case).double()
    for s, x in enumerate(ins):
        keep, age = _row_index(case, s, x["frames"])
        k, v = x["keys"][case["layer"]], x["values"][case["layer"]]
        if keep is not None:
            k, v = k[:, keep], v[:, keep]
        n, n_q = k.shape[1], case["n_q"]
        see = _own_mask(case, seed, s) if case["own"] else None
        if case["op"] == "accumulate":
            w = torch.zeros(case["kv_heads"], x["keys"][0].shape[1], dtype=torch.float64, device=_DEV)
        else:
            out = torch.zeros(case["q_heads"], n_q, case["d"], dtype=torch.float64, device=_DEV)
            lse = torch.zeros(case["q_heads"], n_q, dtype=torch.float64, device=_DEV)
        for g in range(case["kv_heads"]):
            kk, vv = k[g].double(), v[g].double()
            if case["own"]:
                kk = torch.cat([kk, x["own_k"][g, :x["n_own"]].double()])
                vv = torch.cat([vv, x["own_v"][g, :x["n_own"]].double()])
            for h in range(g * G, (g + 1) * G):
                for i0 in range(0, n_q, 128):
                    z = (x["q"][h, i0:i0 + 128].double() * scale) @ kk.t()
                    if case["softcap"]:
                        z = torch.tanh(z / case["softcap"]) * case["softcap"]
                    if case["bias"]:
                        z[:, :n] -= sl[h] * age.double()
                    if case["op"] == "accumulate":
                        t = torch.exp(z - x["lse"][h, i0:i0 + 128, None].double()).sum(0)
                        if keep is None:
                            w[g] += t
                        else:
                            w[g, keep] += t
                        continue
                    if see is not None:
                        z[:, n:][~see[i0:i0 + 128]] = float("-inf")
                    a = torch.logsumexp(z, 1)
                    lse[h, i0:i0 + 128] = a
                    p = torch.exp(z - a[:, None])
                    out[h, i0:i0 + 128] = torch.where(torch.isinf(a)[:, None], 0.0, p) @ vv
        res.append(w if case["op"] == "accumulate" else (out, lse))
    return res


def _exact_evict(case, x):
    """Row by rank: a row stays when fewer than ``keep`` rows of its frame come before it."""
    rows = np.array(_frame_rows(case, x["frames"]))
    first = np.concatenate([[0], np.cumsum(rows)])
    border = max(0, x["frames"] - case["recent"])
    w = x["weights"].double().cpu().numpy()
    stay = np.ones(w.shape, dtype=bool)
    for r in set(rows[:border].tolist()):
        fs = np.nonzero(rows[:border] == r)[0]
        at = first[fs][:, None] + np.arange(r)
        order = np.argsort(-w[:, :, at], axis=-1, kind="stable")
        late = np.take_along_axis(np.broadcast_to(at, order.shape), order[..., case["keep"]:], -1)
        np.put_along_axis(stay, late.reshape(*w.shape[:2], -1), False, -1)
    out = []
    for t in (torch.stack(x["keys"]), torch.stack(x["values"]), x["weights"][..., None]):
        m = torch.from_numpy(stay).to(_DEV)
        y = t[m].reshape(*w.shape[:2], -1, t.shape[-1]).double()
        out.append(y if t.shape[-1] > 1 else y[..., 0])
    return out
