"""Rotation and the paged cache at the ends of what their documentation allows, against the 64-bit
forms of ``paged_ref``."""
import numpy as np
import pytest
import torch

import paged_ref as R
from test_gpu_paged_cache import DEV, Rig, check_attend, check_turn, normal

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------
# the largest values
# --------------------------------------------------------------------------

@pytest.mark.parametrize("heads", [(28, 4, 128), (4, 2, 64)])
@pytest.mark.parametrize("top", [2.0 ** 47, 2.0 ** 48])
def test_values_up_to_the_largest(heads, top):
    """Values at most 2^48, before their block is full and after, by as few query columns as a token has and by many."""
    Hq, Hk, d = heads
    rig = Rig(heads, 1, 4, layers=1, layer=0, seed=61)
    n = 7
    for add in (n, 32 - n, 40):
        k, v = normal(add, Hk, add, d), normal(add + 1, Hk, add, d).clamp(-4, 4)
        v *= top / 4
        v[:, 0, 1], v[:, -1, 0] = top, -top
        rig.lengths += add
        rig.batch.append(0, k.to(DEV), v.to(DEV))
        rig.ref[0].add(k.double(), v.double())
        for q in (1, 5, min(40, rig.ref[0].k.shape[1])):
            check_attend(rig, [q], q=normal(q, Hq, q, d))


# --------------------------------------------------------------------------
# frequencies of another rule
# --------------------------------------------------------------------------

def test_frequencies_written_in_place():
    """Of a ramp over the pairs' indices, in eager calls, appends and replays."""
    import paper_2609_02780_amd as P
    d, n, gain = 64, 5, 1.25
    rot = P.Rotary(d, gain=gain)
    x, pos = normal(1, 3, n, d), torch.tensor([0, 1, 77, 4000, 9])
    dev, at = x.to(DEV), pos.to(DEV)
    rot(dev, at)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = rot(dev, at)
    for scale in (1.0, 0.5):
        f = R.frequencies(d)[0] * (1 - np.linspace(0, 0.9, d // 2)) * scale
        rot.freqs.copy_(torch.from_numpy(f / (2 * np.pi)))
        want = R.rotate(x.double(), pos, f, gain)
        got = rot(dev, at)
        check_turn(got, x.double() * gain, want)
        for _ in range(2):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, got)
        rig = Rig((3, 3, d), 1, 2, layers=1, layer=0)
        k, v = rig.rows(n)
        rig.lengths += n
        assert torch.equal(rig.batch.append(0, k.to(DEV), v.to(DEV), rotary=rot, positions=at, queries=dev), got)


# --------------------------------------------------------------------------
# streams of any lengths
# --------------------------------------------------------------------------

@pytest.mark.parametrize("heads,streams,per", [((8, 8, 128), 64, 1), ((28, 4, 128), 128, 1), ((28, 4, 128), 32, 3),
                                               ((8, 8, 128), 16, 40), ((16, 4, 64), 24, 40), ((28, 4, 128), 5, 90)])
def test_one_long_stream_among_short_and_idle_ones(heads, streams, per):
    """Wide tables, the idle streams side by side, as a padded batch has them, in two orders."""
    width = 300
    rig = Rig(heads, streams, width, layers=1, layer=0, seed=71)
    rng = np.random.default_rng(streams + per)
    long = {0: 33 * 32 + 5, streams // 2: width * 32 + 31}
    rig.add([long.get(s, int(rng.integers(1, 90)) if s < streams * 2 // 3 else 0) for s in range(streams)])
    for window in (0, 9000):
        check_attend(rig, [per] * streams, window=window, uniform=True)
    counts = [int(c) for c in rng.integers(0, per + 1, streams)]
    counts[streams // 2] = per
    check_attend(rig, counts)
    # the same rows in another order of streams
    order = np.roll(np.arange(streams), streams // 2 - 1)
    rig.tables.copy_(rig.tables[torch.from_numpy(order).to(DEV)].clone())
    rig.slots.copy_(rig.slots[torch.from_numpy(order).to(DEV)].clone())
    rig.lengths.copy_(rig.lengths[torch.from_numpy(order).to(DEV)].clone())
    rig.ref = [rig.ref[s] for s in order]
    check_attend(rig, [per] * streams, uniform=True)


@pytest.mark.parametrize("seed", range(4))
def test_shares_of_random_lengths(seed):
    """Lengths and counts of any kind, so that shares end anywhere in a unit and before its first block."""
    rng = np.random.default_rng(seed)
    heads = [(4, 2, 64), (28, 4, 128), (3, 1, 64), (16, 2, 128)][seed]
    streams = [40, 9, 61, 23][seed]
    rig = Rig(heads, streams, 270, layers=1, layer=0, seed=80 + seed)
    kinds = [0, 1, 32, 33, 90, 700, 2500]
    rig.add([int(rng.choice(kinds)) for _ in range(streams)])
    for most in (1, 2, 6, 40):
        counts = [int(c) for c in rng.integers(0, most + 1, streams)]
        counts[0] = most
        check_attend(rig, counts, window=int(rng.choice([0, 2000])))
        check_attend(rig, [most] * streams, uniform=True)


# --------------------------------------------------------------------------
# what p keeps
# --------------------------------------------------------------------------

def _pair_bounds(want, size, top, length, d):
    """How far sums of few terms may be off where each p is kept in at least 11 bits: half a step, 2^-11, of each
    |p v|, the scores' error as in paged_ref.bounds, at most a step of 2^-24 for each token that is added, and the
    output's own rounding to bf16, 2^-8."""
    score = (d + 16) * 2.0 ** -24 * top + 2.0 ** -18
    return size * (2.0 ** -11 + 2 * score[..., None] + length * 2.0 ** -24) + 2.0 ** -8 * want.abs() + 1e-37


@pytest.mark.parametrize("heads", [(28, 4, 128), (16, 4, 64), (3, 1, 64), (8, 8, 128)])
@pytest.mark.parametrize("length", [7, 70, 2490])
def test_p_keeps_eleven_bits(heads, length):
    """Values of 0 but for two tokens of nearly the same weight and opposite values: what is left is small beside either,
    and shows how p was rounded; a wrong or missing row shows as such."""
    Hq, Hk, d = heads
    rig = Rig(heads, 1, 80, layers=1, layer=0, seed=91)
    k, v = normal(length, Hk, length, d), torch.zeros(Hk, length, d, dtype=torch.bfloat16)
    a, b = length // 3, length - 2
    k[:, b] = k[:, a]
    k[:, b, ::16] += 0.0625
    v[:, a], v[:, b] = 448.0, -448.0
    rig.lengths += length
    rig.batch.append(0, k.to(DEV), v.to(DEV))
    rig.ref[0].add(k.double(), v.double())
    hk, hv = rig.ref[0].held()
    coarse = 0
    for n in (1, 4, 8, 36, 70):
        q = normal(n, Hq, n, d)
        out, _ = rig.batch.attend(0, q.to(DEV))
        want, lse, size, top = R.attend(q.double(), hk, hv, length)
        # (a query before the second token sees the first alone, one before both sees neither)
        tol = _pair_bounds(want, size, top, length, d)
        off = (out.cpu().double() - want).abs()
        assert (off <= tol).all(), (n, float((off / tol).max()))
        # p of 8 bits would not do: half a step, 2^-9, of each weight
        z = q.double() @ hk.repeat_interleave(Hq // Hk, 0).transpose(1, 2) / d ** 0.5
        z = z.masked_fill(torch.arange(length) > torch.arange(length - n, length)[:, None], -torch.inf)
        p = torch.exp(z - z.amax(-1, keepdim=True))
        worse = (p.to(torch.bfloat16).double() @ hv.repeat_interleave(Hq // Hk, 0)) / p.sum(-1, keepdim=True)
        coarse += int(((worse.nan_to_num() - want).abs() > tol).sum())
    assert coarse > 0
