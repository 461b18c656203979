"""Rotary positions, a paged cache in 8 bits, and attention over it: the calls
whose speed counts.

Three operators.  Query head h reads KV head h // G.

``rotate``  pairs (a, b) of the first ``dims`` elements of a head become
            g (a cos t - b sin t), g (b cos t + a sin t), t = position * f_i,
            f_i = base^(-2 i / dims); the pairs are (i, i + dims / 2) or
            (2 i, 2 i + 1).  Scaled for long contexts: f_i / factor, or (``original``)
            by parts: with r = original f_i / 2 pi and c = clamp((r - 1) / 31, 0, 1),
            f_i (c + (1 - c) / factor) and g = 1 + 0.1 ln(factor).  Transposed: -sin.
``append``  n new tokens behind the ``old`` ones of each stream.  A token's row is its
            rotated key and its value in bfloat16.  Blocks of 32 tokens that become
            full go to a page of the stream's table in 8 bits (e4m3) with one scale for
            each KV head: a = max(largest magnitude, 2^-100), scale = a / 448, code =
            e4m3(x * (448 / a)).  Rows of the block that is not full stay in bfloat16,
            in one of the stream's two open blocks (block number & 1); so do those of
            the block that the call began in.  Queries are rotated on the way.
``attend``  out = sum_j p_j v_j,  p = softmax of q.k / sqrt(d) over a stream's tokens
            up to the query (the last n tokens are the queries), or the newest ``window``
            of them; the natural log of the normaliser.  ``prior``: the same of an
            earlier call over other rows, with which it is joined.

``listed()`` gives the cases, ``draw(rng)`` one more of the same ranges.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda"
_B = 32                     # tokens of a block


# --------------------------------------------------------------------------
# Cases
# --------------------------------------------------------------------------

def _rotate(name, heads, tokens, d, dims, **kw):
    c = {"name": name, "op": "rotate", "heads": heads, "tokens": tokens, "d": d, "dims": dims, "interleaved": False,
         "factor": 1.0, "original": 0, "first": 0, "spread": False, "token_major": False, "transposed": False}
    c.update(kw)
    return c


def _append(name, heads, streams, n_least, n_most, old_least, old_most, **kw):
    c = {"name": name, "op": "append", "q_heads": heads[0], "kv_heads": heads[1], "d": heads[2], "streams": streams,
         "n_least": n_least, "n_most": n_most, "old_least": old_least, "old_most": old_most, "dims": heads[2],
         "interleaved": False, "factor": 1.0, "original": 0, "queries": True, "token_major": True}
    c.update(kw)
    return c


def _attend(name, heads, streams, n_least, n_most, old_least, old_most, **kw):
    c = {"name": name, "op": "attend", "q_heads": heads[0], "kv_heads": heads[1], "d": heads[2], "streams": streams,
         "n_least": n_least, "n_most": n_most, "old_least": old_least, "old_most": old_most, "window": 0,
         "prior": False, "idle": 0}
    c.update(kw)
    return c


def listed():
    return [
        # one decoded token behind a short text of a tiny model (4/2 heads, d 64): latency
        _attend("attend_token_tiny", (4, 2, 64), 1, 1, 1, 999, 999),
        # one decoded token for each of 64 streams of 1,000 to 16,000 tokens
        _attend("attend_tokens", (28, 4, 128), 64, 1, 1, 1000, 16000),
        # one decoded token over the rows of an hour of frames (3,600 of 196 tokens) and a text
        _attend("attend_token_long", (28, 4, 128), 1, 1, 1, 705633, 705633),
        # a question of 64 tokens over 10 minutes, joined with what it saw of other rows
        _attend("attend_question", (28, 4, 128), 1, 64, 64, 117650, 117650, prior=True),
        # a prompt's last 4,096 tokens of 16,384
        _attend("attend_prompt", (28, 4, 128), 1, 4096, 4096, 12288, 12288),
        # six streams at different stages (1 to 2,000 new tokens), the newest 1,000 tokens seen, d 64
        _attend("attend_ragged", (16, 4, 64), 6, 1, 2000, 0, 5000, window=1000),
        # the next token of one stream of a tiny model
        _append("append_token_tiny", (4, 2, 64), 1, 1, 1, 999, 999, queries=False),
        # the next token of each of 64 streams, their queries rotated on the way
        _append("append_tokens", (28, 4, 128), 64, 1, 1, 1000, 16000),
        # a prompt of 8,192 tokens, positions scaled by parts
        _append("append_prompt", (28, 4, 128), 1, 8192, 8192, 0, 0, factor=4.0, original=4096),
        # one token's queries
        _rotate("rotate_token", 16, 1, 64, 64, first=999),
        # the queries of a prompt far into a stream, as a projection leaves them (token by token)
        _rotate("rotate_prompt", 28, 8192, 128, 128, first=697000, token_major=True, factor=8.0, original=32768),
        # back through a rotation of neighbouring pairs of half the head, tokens of many streams
        _rotate("rotate_back", 16, 1777, 128, 64, interleaved=True, spread=True, first=100000, transposed=True),
    ]


_HEADS = ((4, 2, 64), (16, 4, 64), (16, 2, 128), (28, 4, 128), (8, 8, 128), (16, 1, 128), (3, 1, 64))


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("rotate", "append", "attend", "attend"))
    heads = rng.choice(_HEADS)
    d = heads[2]
    turn = {"interleaved": rng.random() < 0.5, "dims": rng.choice((d, d, d // 2, 2 * rng.randint(1, d // 2)))}
    if rng.random() < 0.5:
        turn["factor"] = rng.choice((2.0, 4.0, 8.0, 2.5))
        turn["original"] = rng.choice((0, 4096, 8192, 32768))
    if op == "rotate":
        c = _rotate("", rng.choice((1, heads[1], heads[0])), _log_int(rng, 1, 8192), d, d, first=_log_int(rng, 1, 1000000),
                    spread=rng.random() < 0.3, token_major=rng.random() < 0.5, transposed=rng.random() < 0.5)
        c.update(turn)
    elif op == "append":
        many = rng.random() < 0.5
        n = _log_int(rng, 1, 8 if many else 8192)
        old = _log_int(rng, 1, 20000)
        c = _append("", heads, _log_int(rng, 2, 64) if many else rng.randint(1, 3), rng.choice((n, 1)), n,
                    rng.choice((old, 0)), old, queries=rng.random() < 0.6, token_major=rng.random() < 0.6)
        c.update(turn)
    else:
        kind = rng.choice(("token", "token", "drafts", "prompt"))
        n = {"token": 1, "drafts": rng.randint(2, 100), "prompt": _log_int(rng, 100, 4096)}[kind]
        S = 1 if rng.random() < 0.4 else _log_int(rng, 2, 64 if kind == "token" else 8)
        old = _log_int(rng, 1, 700000)
        c = _attend("", heads, S, rng.choice((n, 1)), n, rng.choice((old, old // 2, 0)), old,
                    window=rng.choice((0, 0, _log_int(rng, 1, 20000))), prior=rng.random() < 0.3,
                    idle=rng.choice((0, 0, S // 3)))
    del c["name"]
    top = [work(x) for x in listed()]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    while any(work(c)[k] > most[k] for k in most) or _padded(c) > 4e8:
        for k in ("old_most", "n_most"):
            c[k] = max(1, c[k] * 2 // 3)
        c["old_least"], c["n_least"] = min(c["old_least"], c["old_most"]), min(c["n_least"], c["n_most"])
    return c


def _padded(case):
    """Values of the plain form's padded rows and scores: a bound on its memory."""
    if case["op"] != "attend":
        return 0
    n, L = max(_new(case)), max(_lengths(case)) + _B
    return case["streams"] * L * max(case["kv_heads"] * case["d"], case["q_heads"] * n / 8)


def _spread(lo, hi, S, k):
    """S numbers from lo to hi in a mixed order, both ends among them."""
    return [hi] if S == 1 else [lo + (hi - lo) * ((s * k) % S if S % k else s) // (S - 1) for s in range(S)]


def _new(case):
    """New tokens (queries) of each stream."""
    return _spread(case["n_least"], case["n_most"], case["streams"], 3)


def _lengths(case):
    """Tokens of each stream, the new ones among them; none for an idle stream."""
    idle = case.get("idle", 0)
    out = []
    for s, (n, old) in enumerate(zip(_new(case), _spread(case["old_least"], case["old_most"], case["streams"], 5))):
        if case["op"] == "append":
            # over an even number of blocks a call ends in the open block that it began in: then it begins a block,
            # so that a pass finds what the pass before it found
            if ((old + n - 1) // _B - old // _B) % 2 == 0 and (old + n - 1) // _B > old // _B:
                old -= old % _B
        out.append(0 if s < idle else old + n)
    return out


def _freqs(case):
    """f_i in 64 bits and the gain."""
    D = case["dims"]
    f = 10000.0 ** (-2.0 * np.arange(D // 2) / D)
    gain = 1.0
    if case["factor"] != 1.0:
        if case["original"]:
            c = np.clip((case["original"] * f / (2.0 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
            f = f * (c + (1.0 - c) / case["factor"])
            gain = 1.0 + 0.1 * math.log(case["factor"])
        else:
            f = f / case["factor"]
    return f, gain


def work(case):
    d = case["d"]
    if case["op"] == "rotate":
        return {"bytes": case["tokens"] * (case["heads"] * d * 4 + 8), "flops": 3 * case["heads"] * case["tokens"] * case["dims"]}
    Hq, Hk = case["q_heads"], case["kv_heads"]
    total_b = total_f = 0
    for n, L in zip(_new(case), _lengths(case)):
        old = L - n
        if case["op"] == "append":
            full = L // _B - old // _B
            total_b += Hk * (n * 4 * d + full * (2 * _B * d + 8)) + n * 8
            if full:                                                     # the earlier rows of the first block
                total_b += Hk * (old % _B) * 4 * d
            total_b += Hk * (L % _B if full else n) * 4 * d              # rows of the open block
            total_f += 3 * Hk * n * case["dims"]
            if case["queries"]:
                total_b += Hq * n * 4 * d
                total_f += 3 * Hq * n * case["dims"]
            continue
        if L == 0:
            total_b += Hq * n * (2 * d + 4)
            continue
        w = case["window"] or L + 1
        lo = max(0, old + 1 - w)                                         # the first token that any query sees
        full = L // _B - lo // _B
        total_b += Hk * (full * (2 * _B * d + 8) + L % _B * 4 * d) + Hq * n * (4 * d + 4)
        if case["prior"]:
            total_b += Hq * n * (2 * d + 4)
        # query i sees min(w, old + i + 1) tokens
        k = min(max(0, w - old - 1), n)
        pairs = k * old + k * (k + 1) // 2 + (n - k) * w
        total_f += 4 * Hq * d * pairs
    return {"bytes": total_b, "flops": total_f}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _normal(gen, *shape, scale=1.0):
    return torch.randn(*shape, generator=gen, device=_DEV, dtype=torch.bfloat16) * scale


def _rows(gen, case, key, *shape):
    """Rows of keys or values: keys have a few strong dimensions."""
    x = _normal(gen, *shape)
    if key:
        strong = torch.ones(shape[-1], device=_DEV, dtype=torch.bfloat16)
        strong[3::29] = 4.0
        x = x * strong * 0.7
    return x


def _heads_of(gen, case, key, heads, n):
    """[heads][n][d], token by token in memory or head by head."""
    if case["token_major"]:
        return _rows(gen, case, key, n, heads, case["d"]).transpose(0, 1)
    return _rows(gen, case, key, heads, n, case["d"])


def _positions(case, seed):
    """int64 [tokens] of a rotation."""
    n, first = case["tokens"], case["first"]
    if case["spread"]:
        return torch.from_numpy(np.random.default_rng([seed, 5]).integers(0, first + n, n)).to(_DEV)
    return first + torch.arange(n, device=_DEV)


def _inputs(case, seed):
    """Everything that a call is given and the cache before it; the same for every form."""
    gen = torch.Generator(device=_DEV)
    gen.manual_seed(seed * 1009 + 3)
    x = {}
    if case["op"] == "rotate":
        x["x"] = _heads_of(gen, case, False, case["heads"], case["tokens"])
        x["positions"] = _positions(case, seed)
        return x
    S, Hq, Hk, d = case["streams"], case["q_heads"], case["kv_heads"], case["d"]
    n, L = _new(case), _lengths(case)
    N = sum(n)
    need = [v // _B for v in L]
    W = max(1, max(need))
    P = max(1, sum(need)) + 3
    rng = np.random.default_rng([seed, 11])
    at = rng.permutation(P)
    table = np.zeros((S, W), dtype=np.int32)
    for s, k in enumerate(need):
        table[s, :k], at = at[:k], at[k:]
    x["tables"] = torch.from_numpy(table).to(_DEV)
    x["lengths"] = torch.tensor(L, dtype=torch.int32, device=_DEV)
    slots = rng.permutation(S + 2)[:S].astype(np.int32)
    x["slots"] = torch.from_numpy(slots).to(_DEV)
    for name in ("keys", "values"):
        rows = _rows(gen, case, name == "keys", P, Hk, _B, d).float()
        a = rows.abs().amax((2, 3), keepdim=True)
        x["page_" + name] = (rows * (448.0 / a)).to(torch.float8_e4m3fn)
        x[name + "_scale"] = (a / 448.0)[:, :, 0, 0].contiguous()
        x["open_" + name] = _rows(gen, case, name == "keys", S + 2, 2, Hk, _B, d)
        del rows
    if case["op"] == "append":
        x["keys"] = _heads_of(gen, case, True, Hk, N)
        x["values"] = _heads_of(gen, case, False, Hk, N)
        if case["queries"]:
            x["q"] = _heads_of(gen, case, False, Hq, N)
        return x
    x["q"] = _normal(gen, Hq, N, d, scale=1.5)
    if case["prior"]:
        x["prior_out"] = _normal(gen, Hq, N, d, scale=0.2)
        x["prior_lse"] = math.log(max(1, max(L))) + 1.0 + torch.randn(Hq, N, generator=gen, device=_DEV)
    return x


def _key_rows(t):
    """[...][32][d] as the cache's views of keys have it: [...][32][d / 16][16]."""
    return t.unflatten(-1, (t.shape[-1] // 16, 16))


def _value_rows(t):
    """[...][32][d] as the cache's views of values have it: [...][2][2][2][4][d / 32][32]."""
    return t.unflatten(-1, (t.shape[-1] // 32, 32)).unflatten(-3, (2, 2, 2, 4))


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["op"] != "attend":
        f, st["gain"] = _freqs(case)
        st["freqs"] = torch.from_numpy(f).to(_DEV)
    if not own:
        return st
    import paper_2609_02780_amd as P
    if case["op"] != "attend":
        st["rotary"] = P.Rotary(case["dims"], interleaved=case["interleaved"], factor=case["factor"],
                                original=case["original"])
    if case["op"] == "rotate":
        return st
    st["n"] = _new(case) if case["n_least"] != case["n_most"] else None
    cache = P.PagedCache(1, case["q_heads"], case["kv_heads"], case["d"], st["page_keys"].shape[0],
                         st["open_keys"].shape[0])
    cache.keys[0].copy_(_key_rows(st.pop("page_keys")))
    cache.values[0].copy_(_value_rows(st.pop("page_values")))
    cache.key_scales[0].copy_(st.pop("keys_scale"))
    cache.value_scales[0].copy_(st.pop("values_scale"))
    cache.open_keys[0].copy_(_key_rows(st.pop("open_keys")))
    cache.open_values[0].copy_(_value_rows(st.pop("open_values")))
    st["cache"] = cache
    st["batch"] = P.PagedBatch(cache, st["tables"], st["lengths"], st["slots"])
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        return _run_own(case, state)
    if case["op"] == "rotate":
        return _plain_turn(case, state, state["x"], state["positions"], case["transposed"]).to(torch.bfloat16)
    if case["op"] == "append":
        return _plain_append(case, state)
    return _plain_attend(case, state)


def _run_own(case, st):
    if case["op"] == "rotate":
        return st["rotary"](st["x"], st["positions"], transposed=case["transposed"])
    if case["op"] == "append":
        q = st["batch"].append(0, st["keys"], st["values"], n_new=st["n"], rotary=st["rotary"], queries=st.get("q"))
        c = st["cache"]
        return {"q": q, "keys": c.keys[0], "values": c.values[0], "key_scales": c.key_scales[0],
                "value_scales": c.value_scales[0], "open_keys": c.open_keys[0], "open_values": c.open_values[0]}
    return st["batch"].attend(0, st["q"], n_q=st["n"], window=case["window"],
                              prior=(st["prior_out"], st["prior_lse"]) if case["prior"] else None)


def _plain_turn(case, st, x, positions, back=False):
    """Rotated [H][N][d] in 32 bits; angles in 64 (far positions)."""
    D = case["dims"]
    t = positions.double()[:, None] * st["freqs"]
    c, s = (torch.cos(t) * st["gain"]).float(), (torch.sin(t) * (-st["gain"] if back else st["gain"])).float()
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:D:2], y[..., 1:D:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = y[..., :D // 2], y[..., D // 2:D]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, y[..., D:]], -1)


def _stream_of(case):
    """Each new token's stream and its place among the stream's new tokens."""
    n = torch.tensor(_new(case), device=_DEV)
    sid = torch.repeat_interleave(torch.arange(case["streams"], device=_DEV), n, output_size=sum(_new(case)))
    start = torch.cumsum(n, 0) - n
    return n, start, sid, torch.arange(sid.shape[0], device=_DEV) - start[sid]


def _plain_append(case, st):
    n, start, sid, i = _stream_of(case)
    L = st["lengths"].long()
    old = L - n
    at = old[sid] + i
    rows = {"keys": _plain_turn(case, st, st["keys"], at).to(torch.bfloat16), "values": st["values"]}
    # blocks that are full now
    nb = L // _B - old // _B
    sb = torch.repeat_interleave(torch.arange(case["streams"], device=_DEV), nb)
    b = (old // _B)[sb] + torch.arange(sb.shape[0], device=_DEV) - (torch.cumsum(nb, 0) - nb)[sb]
    t = b[:, None] * _B + torch.arange(_B, device=_DEV)
    new = t >= old[sb, None]
    src = (start[sb, None] + t - old[sb, None]).clamp(0, sid.shape[0] - 1)
    page = st["tables"].long()[sb, b]
    # rows that stay as they are: those of the last block, and of the first where it has an open block of its own
    last, bt = ((L - 1) // _B)[sid], at // _B
    keep = torch.nonzero((bt == last) | ((bt == old[sid] // _B) & ((last - bt) % 2 == 1))).flatten()
    slot = st["slots"].long()
    for name in ("keys", "values"):
        r, open_ = rows[name], st["open_" + name]
        block = torch.where(new[:, None, :, None], r[:, src].transpose(0, 1), open_[slot[sb], b & 1]).float()
        a = block.abs().amax((2, 3)).clamp_min(2.0 ** -100)
        st["page_" + name][page] = (block * (448.0 / a)[:, :, None, None]).to(torch.float8_e4m3fn)
        st[name + "_scale"][page] = a / 448.0
        open_[slot[sid[keep]], bt[keep] & 1, :, at[keep] % _B] = r[:, keep].transpose(0, 1)
    q = _plain_turn(case, st, st["q"], at).to(torch.bfloat16) if case["queries"] else None
    return {"q": q, "keys": _key_rows(st["page_keys"]), "values": _value_rows(st["page_values"]),
            "key_scales": st["keys_scale"], "value_scales": st["values_scale"],
            "open_keys": _key_rows(st["open_keys"]), "open_values": _value_rows(st["open_values"])}


def _plain_rows(st, name, full):
    """A stream's rows in 32 bits, [S][H][W 32 + 32][d]: its pages, then its open block."""
    S, W = st["tables"].shape
    page = st["tables"].long()
    x = st["page_" + name][page].float() * st[name + "_scale"][page][..., None, None]
    x = x.permute(0, 2, 1, 3, 4).flatten(2, 3)
    return torch.cat([x, st["open_" + name][st["slots"].long(), full & 1].float()], 2)


def _plain_attend(case, st):
    S, Hq, Hk, d = case["streams"], case["q_heads"], case["kv_heads"], case["d"]
    G = Hq // Hk
    n, start, sid, i = _stream_of(case)
    most = max(_new(case))
    L = st["lengths"].long()
    full = L // _B
    k, v = _plain_rows(st, "keys", full), _plain_rows(st, "values", full)
    W = st["tables"].shape[1] * _B
    # each row's token, none behind the stream's end
    j = torch.arange(W + _B, device=_DEV)
    tok = torch.where(j < W, j, full[:, None] * _B + j - W)
    there = torch.where(j < W, j < full[:, None] * _B, tok < L[:, None])
    qi = (start[:, None] + torch.arange(most, device=_DEV)).clamp(max=sid.shape[0] - 1)
    qp = (L - n)[:, None] + torch.arange(most, device=_DEV)
    see = there[:, None] & (tok[:, None] <= qp[..., None])
    if case["window"]:
        see &= tok[:, None] > qp[..., None] - case["window"]
    q = st["q"][:, qi].float().reshape(Hk, G, S, most, d).permute(2, 0, 1, 3, 4).reshape(S, Hk, G * most, d)
    sc = torch.matmul(q * (1.0 / math.sqrt(d)), k.transpose(2, 3).contiguous()).reshape(S, Hk, G, most, -1)
    sc = sc.masked_fill(~see[:, None, None], float("-inf"))
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    p = torch.exp(sc - top)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(S, Hk, G * most, -1), v).reshape(S, Hk, G, most, d)
    o = torch.where(z > 0, o / z, torch.zeros_like(o))
    lse = (top + torch.log(z))[..., 0]
    # back to the tokens' order
    o = o.permute(1, 2, 0, 3, 4).reshape(Hq, S, most, d)[:, sid, i]
    lse = lse.permute(1, 2, 0, 3).reshape(Hq, S, most)[:, sid, i]
    if case["prior"]:
        both = torch.logaddexp(lse, st["prior_lse"])
        o = torch.exp(lse - both)[..., None] * o + torch.exp(st["prior_lse"] - both)[..., None] * st["prior_out"].float()
        lse = both
    return o.to(torch.bfloat16), lse


# --------------------------------------------------------------------------
# The definition in 64 bits
# --------------------------------------------------------------------------

def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "rotate":
        return _exact_turn(case, x["x"], x["positions"].cpu().numpy(), case["transposed"])
    return _exact_append(case, x) if case["op"] == "append" else _exact_attend(case, x)


def _exact_turn(case, x, positions, back=False):
    """Each pair as a complex number times gain e^(i t)."""
    f, gain = _freqs(case)
    D = case["dims"]
    t = positions[:, None] * f
    w = torch.from_numpy(gain * np.exp((-1j if back else 1j) * t)).to(_DEV)
    y = x.double().clone()
    pick = [torch.arange(0, D, 2), torch.arange(1, D, 2)] if case["interleaved"] else \
        [torch.arange(D // 2), torch.arange(D // 2, D)]
    z = torch.complex(y[..., pick[0].to(_DEV)], y[..., pick[1].to(_DEV)]) * w
    y[..., pick[0].to(_DEV)], y[..., pick[1].to(_DEV)] = z.real, z.imag
    return y


def _to_e4m3(y):
    """The nearest of the values with 3 bits behind the point (ties to even), down to multiples of 2^-9, up to 448."""
    e = torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -40))).clamp_min(-6.0)
    step = torch.exp2(e - 3.0)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)


def _exact_append(case, x):
    n, L = _new(case), _lengths(case)
    table, slot = x["tables"].cpu().numpy(), x["slots"].cpu().numpy()
    at = np.concatenate([np.arange(l - k, l) for k, l in zip(n, L)])
    turned = _exact_turn(case, x["keys"], at)
    res = {"q": _exact_turn(case, x["q"], at) if case["queries"] else None}
    for name, rows in (("keys", turned.float().to(torch.bfloat16).double()), ("values", x["values"].double())):
        pages, open_ = x["page_" + name].float().double(), x["open_" + name].double()
        scales = x[name + "_scale"].double()
        first = 0
        for s in range(case["streams"]):
            old = L[s] - n[s]
            b0, b1 = old // _B, (L[s] - 1) // _B
            # the stream's rows from its first touched block on
            all_ = torch.cat([open_[slot[s], b0 & 1, :, :old % _B], rows[:, first:first + n[s]]], 1)
            first += n[s]
            for b in range(b0, L[s] // _B):
                blk = all_[:, (b - b0) * _B:(b - b0 + 1) * _B]
                a = blk.abs().amax((1, 2)).clamp_min(2.0 ** -100)
                pages[table[s, b]] = _to_e4m3(blk * (448.0 / a)[:, None, None])
                scales[table[s, b]] = a / 448.0
            for b in sorted({b0, b1}):            # the later block has the last word
                blk = all_[:, (b - b0) * _B:(b - b0 + 1) * _B]
                if b == b1 or (b1 - b) % 2:
                    open_[slot[s], b & 1, :, :blk.shape[1]] = blk
        as_rows = _key_rows if name == "keys" else _value_rows
        res[name], res["open_" + name] = as_rows(pages), as_rows(open_)
        res["key_scales" if name == "keys" else "value_scales"] = scales
    return res


def _exact_attend(case, x):
    Hq, Hk, d = case["q_heads"], case["kv_heads"], case["d"]
    G = Hq // Hk
    n, L = _new(case), _lengths(case)
    N = sum(n)
    out = torch.zeros(Hq, N, d, dtype=torch.float64, device=_DEV)
    lse = torch.full((Hq, N), -math.inf, dtype=torch.float64, device=_DEV)
    first = 0
    for s in range(case["streams"]):
        full, tail = divmod(L[s], _B)
        page = x["tables"][s, :full].long()
        for g in range(Hk):
            kv = []
            for name in ("keys", "values"):
                t = (x["page_" + name][page, g].float().double() * x[name + "_scale"][page, g].double()[:, None, None])
                kv.append(torch.cat([t.flatten(0, 1), x["open_" + name][x["slots"][s].long(), full & 1, g, :tail].double()]))
            for i0 in range(0, n[s] if L[s] else 0, 512):
                i1 = min(n[s], i0 + 512)
                last = torch.arange(L[s] - n[s] + i0, L[s] - n[s] + i1, device=_DEV)
                j = torch.arange(L[s], device=_DEV)
                hide = j > last[:, None]
                if case["window"]:
                    hide |= j <= last[:, None] - case["window"]
                for h in range(g * G, (g + 1) * G):
                    z = (x["q"][h, first + i0:first + i1].double() @ kv[0].t()) / math.sqrt(d)
                    z[hide] = -math.inf
                    a = torch.logsumexp(z, 1)
                    p = torch.exp(z - torch.where(torch.isinf(a), 0.0, a)[:, None])
                    out[h, first + i0:first + i1], lse[h, first + i0:first + i1] = p @ kv[1], a
        first += n[s]
    if case["prior"]:
        pl = x["prior_lse"].double()
        m = torch.maximum(lse, pl)
        wa, wb = torch.exp(lse - m), torch.exp(pl - m)
        out = (out * wa[..., None] + x["prior_out"].double() * wb[..., None]) / (wa + wb)[..., None]
        lse = m + torch.log(wa + wb)
    return out, lse
