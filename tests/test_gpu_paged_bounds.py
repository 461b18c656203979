"""The paged cache at the ends of what its documentation allows: the largest values, against the
64-bit forms of ``paged_ref``."""
import pytest
import torch

import paged_ref as R
from test_gpu_paged_cache import DEV, Rig, check_attend, normal

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
