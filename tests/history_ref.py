"""Attention over stored rows, its row weights and eviction in 64 bits (NumPy), with
error bounds for a kernel that forms scores, maxima and sums in fp32 and rounds the
probabilities and the output to bfloat16.

Bounds count roundings of at most u = 2^-24 (fp32) and h = 2^-8 (bfloat16), relative:
  score   q.k adds d products: (d + 2) u sum|q_e k_e| / sqrt(d); scaling, cap, bias and
          the shift by the maximum add a few u of each magnitude (8 u, and 32 u of a
          capped score for its tanh);
  p       exp of a score that is off by e is off by e relative (2 e bounds e^e - 1 here),
          one bfloat16 rounding: h;
  flush   a p below the smallest normal fp32 number, 2^-126, may come out as 0: each of the
          terms of a weight, the only sums that are not taken against a maximum, is then off
          by less than 2^-126 (far rows under a steep bias have weights of 1e-80);
  sums    n terms of one sign added in any order: at most n u relative, a tree or lane
          split only fewer; the maximum's rescaling adds one rounding a tile;
  out     a weighted mean of the values: each relative error r of the p's moves it by at
          most 2 r sum p|v|, of which the bfloat16 one reaches the numerator only (h);
          its own rounding adds h |out|.
"""
import numpy as np

U = 2.0 ** -24
H = 2.0 ** -8


def f64(bits):
    return (np.ascontiguousarray(bits).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def scores(q, k, softcap, slope, age):
    """Scores [n_q][n] of one head, and a bound of their fp32 error."""
    d = q.shape[1]
    s = q @ k.T / np.sqrt(d)
    err = (d + 2) * U * (np.abs(q) @ np.abs(k).T) / np.sqrt(d) + 8 * U * np.abs(s)
    if softcap:
        s = softcap * np.tanh(s / softcap)
        err = err + 32 * U * np.abs(s)
    if slope is not None:
        b = slope * age
        s = s - b[None, :]
        err = err + 8 * U * np.abs(b)[None, :]
    return s, err


def attend(q, k, v, mask, G, softcap=0.0, slopes=None, age=None):
    """q [H_q][n_q][d], k and v [H_kv][n][d], mask [n_q][n], age [n].  Returns out, lse
    and a bound of the error of each."""
    Hq, nq, d = q.shape
    n = k.shape[1]
    out, lse = np.zeros((Hq, nq, d)), np.full((Hq, nq), -np.inf)
    b_out, b_lse = np.zeros((Hq, nq, d)), np.zeros((Hq, nq))
    if n == 0:
        return out, lse, b_out, b_lse
    for h in range(Hq):
        s, err = scores(q[h], k[h // G], softcap, None if slopes is None else slopes[h], age)
        s = np.where(mask, s, -np.inf)
        m = s.max(1, keepdims=True)
        p = np.exp(s - np.where(np.isinf(m), 0.0, m))
        z = p.sum(1)
        e = np.where(mask, err, 0.0).max(1) + 8 * U * np.abs(np.where(np.isinf(m), 0.0, m))[:, 0] + 4 * U
        live = z > 0
        pn = np.where(live[:, None], p / np.where(live, z, 1.0)[:, None], 0.0)
        out[h] = pn @ v[h // G]
        mag = pn @ np.abs(v[h // G])
        lse[h] = np.where(live, np.where(np.isinf(m), 0, m)[:, 0] + np.log(np.where(live, z, 1.0)), -np.inf)
        rel = 2 * e + (n + 64) * U
        b_out[h] = (H + 2 * rel)[:, None] * mag + H * np.abs(out[h]) * (1 + H) + 1e-30
        b_lse[h] = rel + 8 * U * (np.abs(np.where(live, lse[h], 0.0)) + 1)
    return out, lse, b_out, b_lse


def weights(q, k, lse, G, softcap=0.0, slopes=None, age=None):
    """sum over heads and queries of exp(s - lse), [H_kv][n], and its bound."""
    Hq, nq, _ = q.shape
    w, b = np.zeros(k.shape[:2]), np.full(k.shape[:2], G * nq * 2.0 ** -126)
    for h in range(Hq):
        s, err = scores(q[h], k[h // G], softcap, None if slopes is None else slopes[h], age)
        z = np.asarray(lse[h], dtype=np.float64)
        live = ~np.isinf(z)
        zz = np.where(live, z, 0.0)[:, None]
        p = np.where(live[:, None], np.exp(s - zz), 0.0)
        w[h // G] += p.sum(0)
        b[h // G] += (p * (2 * (err + 8 * U * (np.abs(s) + np.abs(zz))) + (Hq * nq + 8) * U)).sum(0)
    return w, b


def causal(n_q, n_own):
    """[n_q][n_own]: the queries are the last own tokens."""
    return np.arange(n_own)[None, :] <= (n_own - n_q + np.arange(n_q))[:, None]


def tree_mask(parents, n_own):
    n = len(parents)
    m = np.zeros((n, n_own), dtype=bool)
    m[:, :n_own - n] = True
    for i in range(n):
        j = i
        while True:
            m[i, n_own - n + j] = True
            p = int(parents[j])
            if not 0 <= p < j:
                break
            j = p
    return m


def kept_rows(w, rows, n_thin, keep):
    """Positions kept by one (layer, KV head): w [n], rows per frame."""
    out, lo = [], 0
    for f, r in enumerate(rows):
        pos = np.arange(lo, lo + r)
        if f < n_thin and keep < r:
            order = sorted(range(r), key=lambda i: (-float(w[lo + i]), i))[:keep]
            pos = lo + np.array(sorted(order), dtype=np.int64)
        out.append(pos)
        lo += r
    return np.concatenate(out) if out else np.zeros(0, dtype=np.int64)
