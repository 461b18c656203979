"""Rotation and the paged cache at the ends of what their documentation allows, against the 64-bit
forms of ``paged_ref``."""
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
    import numpy as np

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
