"""Rotary positions and the paged cache in 64 bits on the CPU, from their definitions."""
import math

import numpy as np
import torch

BLOCK = 32


def frequencies(dims, base=10000.0, factor=1.0, original=0.0, fast=32.0, slow=1.0):
    """Radians a position, and the gain."""
    f = base ** (-2.0 * np.arange(dims // 2) / dims)
    if original > 0 and factor > 1:
        c = np.clip((original * f / (2 * math.pi) - slow) / (fast - slow), 0, 1)
        return f * (c + (1 - c) / factor), 1 + 0.1 * math.log(factor)
    return f / factor, 1.0


def rotate(x, positions, freqs, gain=1.0, interleaved=False, transposed=False):
    """x [H][N][d] float64; positions a sequence of N whole numbers."""
    D = 2 * len(freqs)
    t = np.asarray(positions, dtype=np.float64)[:, None] * freqs
    c, s = torch.from_numpy(np.cos(t) * gain), torch.from_numpy(np.sin(t) * gain * (-1 if transposed else 1))
    y = x.clone()
    ia, ib = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    a, b = x[..., ia], x[..., ib]
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    return y


def quantised(block):
    """A block's rows [H][32][d] (bf16 values in any type) -> codes (float8) and scales, by the definition's fp32 steps."""
    x = block.float()
    a = x.abs().amax((1, 2)).clamp_min(2.0 ** -100)
    # (448.0 / tensor would be two roundings, a reciprocal and a product)
    inverse = torch.full_like(a, 448.0).div(a)
    return (x * inverse[:, None, None]).to(torch.float8_e4m3fn), a / 448.0


class Stream:
    """A stream's rows (bf16 values, float64 [H][n][d]) and what a cache holds of them."""

    def __init__(self, heads, d):
        self.k = torch.zeros(heads, 0, d, dtype=torch.float64)
        self.v = torch.zeros(heads, 0, d, dtype=torch.float64)

    def add(self, k, v):
        self.k, self.v = torch.cat([self.k, k], 1), torch.cat([self.v, v], 1)

    def held(self):
        """Keys and values as the cache stands for them."""
        out = []
        for x in (self.k, self.v):
            y = x.clone()
            for b in range(x.shape[1] // BLOCK):
                at = slice(b * BLOCK, (b + 1) * BLOCK)
                codes, scale = quantised(x[:, at])
                y[:, at] = codes.double() * scale.double()[:, None, None]
            out.append(y)
        return out

    def value_steps(self):
        """What a value is counted in, [H][n]: the scale of a full block, the power of two that lifts the largest of
        an open one to 2^7."""
        out, n = [], self.v.shape[1]
        for b in range(0, n, BLOCK):
            x = self.v[:, b:b + BLOCK]
            if x.shape[1] == BLOCK:
                s = quantised(x)[1].double()
            else:
                s = 2.0 ** (torch.floor(torch.log2(x.abs().amax((1, 2)).clamp_min(2.0 ** -57))) - 7)
            out.append(s.clamp_min(2.0 ** -64)[:, None].expand(-1, x.shape[1]))
        return torch.cat(out, 1) if out else torch.zeros(self.v.shape[0], 0, dtype=torch.float64)


def attend(q, k, v, length, window=0, seen=None, prior=None, steps=None):
    """q [Hq][n][d] float64, the last n of `length` tokens; k, v [Hk][length][d].  seen: truth of each
    token; steps: Stream.value_steps().  Returns out, lse, and for bounds sum p |v| and the largest sum |q_i k_i| / sqrt(d)."""
    Hq, n, d = q.shape
    G = Hq // k.shape[0]
    kk, vv = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    at = torch.arange(length - n, length)[:, None]
    j = torch.arange(length)
    hide = j > at
    if window:
        hide = hide | (j <= at - window)
    if seen is not None:
        hide = hide | ~seen
    z = (q @ kk.transpose(1, 2)) / math.sqrt(d)
    z = z.masked_fill(hide, -math.inf)
    mass = (q.abs() @ kk.abs().transpose(1, 2) / math.sqrt(d)).masked_fill(hide, 0.0)
    lse = torch.logsumexp(z, -1) if length else torch.full((Hq, n), -math.inf, dtype=torch.float64)
    p = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
    out, size = p @ vv, p @ vv.abs()
    if steps is not None and length:
        # p times its step is kept in 11 bits or steps of 2^-33 of the largest such product: off by 2^-34 of it
        # for each seen value, in its step.  bounds() multiplies by 2^-8
        w = steps.repeat_interleave(G, 0)
        size = size + 2.0 ** -26 * (p * w[:, None]).amax(-1, keepdim=True) * ((p > 0).double() @ (vv.abs() / w[..., None]))
    top = mass.amax(-1) if length else torch.zeros(Hq, n, dtype=torch.float64)
    if prior is not None:
        po, pl = prior
        m = torch.maximum(lse, pl)
        m = torch.where(torch.isinf(m), 0.0, m)
        wa, wb = torch.exp(lse - m), torch.exp(pl - m)
        z = torch.where(wa + wb > 0, wa + wb, 1.0)
        po = torch.where((wb > 0)[..., None], po, 0.0)
        out = (out * wa[..., None] + po * wb[..., None]) / z[..., None]
        size = (size * wa[..., None] + po.abs() * wb[..., None]) / z[..., None]
        lse = m + torch.log(wa + wb)
    return out, lse, size, top


def bounds(out, lse, size, top, d):
    """How far an output may be off.  p and the output are rounded to bf16, half a step (2^-8 of the value)
    each; a score is a chain of d fp32 sums of exact products and a few fp32 steps, so it is off by
    (d + 16) 2^-24 of its terms' sum, which is p's and lse's relative error; exp and the sums in fp32
    add some 2^-18."""
    score = (d + 16) * 2.0 ** -24 * top + 2.0 ** -18
    return (2.0 ** -8 * (1 + 2.0 ** -7)) * (size + out.abs()) + 2 * score[..., None] * size + 1e-37, \
        score + 2.0 ** -22 * torch.where(torch.isinf(lse), 0.0, lse.abs())
