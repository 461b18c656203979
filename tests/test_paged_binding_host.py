"""What the paged cache's binding holds for its calls cannot be exchanged beside them.  No GPU."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def P():
    from paper_2609_02780_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_02780_amd.build import build_library
        build_library()
    import paper_2609_02780_amd
    return paper_2609_02780_amd


def test_a_rotation_is_what_its_attributes_say(P):
    """Calls take the address of the frequencies, the gain and the pairs that a rotation was made with: none is
    replaced, frequencies are written where they lie."""
    rot = P.Rotary(64, interleaved=True, factor=4.0, original=256, device="cpu")
    held, at = rot.freqs, rot._c.freqs
    assert (rot.dims, rot.interleaved) == (64, True) and rot.gain == rot._c.gain > 1.1
    with pytest.raises(ValueError, match="in place"):
        rot.freqs = torch.ones(32, dtype=torch.float64)
    for name, value in (("gain", 1.0), ("dims", 32), ("interleaved", False)):
        with pytest.raises(AttributeError):
            setattr(rot, name, value)
    want = held / 3
    rot.freqs /= 3
    assert rot.freqs is held and torch.equal(held, want)
    rot.freqs.copy_(torch.arange(32) / 64)
    assert rot._c.freqs == at == held.data_ptr()
    assert P.Rotary(64, gain=2.5, device="cpu").gain == 2.5


def test_a_batch_stays_with_its_cache(P):
    """Sizes of outputs and workspaces are kept by a batch and hold for its cache's heads alone."""
    from types import SimpleNamespace
    ints = torch.zeros(2, dtype=torch.int32)
    cache, other = (SimpleNamespace(arena=torch.empty(1)) for _ in range(2))
    batch = P.PagedBatch(cache, ints.reshape(2, 1), ints, ints)
    with pytest.raises(AttributeError):
        batch.cache = other
    assert batch.cache is cache
