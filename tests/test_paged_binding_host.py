"""The paged cache on the host: what its binding holds for its calls cannot be exchanged beside them, and how
attention is cut, by the workspaces that it asks for.  No GPU."""
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


@pytest.mark.parametrize("heads,streams,tokens", [((28, 4, 128), 128, 1), ((28, 4, 128), 256, 1), ((28, 4, 128), 512, 1), ((8, 8, 128), 64, 1),
                                                  ((28, 4, 128), 128, 10), ((28, 4, 128), 32, 64), ((16, 2, 128), 4, 1024)])
def test_streams_that_may_differ_are_shared(P, heads, streams, tokens):
    """The tables' width stands for every stream's length, but streams of any lengths may be long alone: then no
    unit is one thread block's, however well as many equal ones would fill the card.  Shares take a workspace."""
    import ctypes as C

    from paper_2609_02780_amd import _lib as L
    fake, h = 0x7F0000000000, C.c_void_p()
    d = L.CacheDesc(1, *heads, 10, 600)
    assert L.lib().ss_cache_create(C.byref(d), fake, 1 << 60, C.byref(h)) == 0
    need = lambda width, window=0: L.lib().ss_cache_attend_workspace_bytes(        # noqa: E731
        h, C.byref(L.CacheStreams(fake, fake, fake, streams, width)), streams * tokens, None, window)
    for width in (300, 500, 2000, 20000):
        assert need(width) > 256, width
    # short ones are not worth joining
    assert need(20) == need(20000, 100) == 256
    assert L.lib().ss_cache_destroy(h) == 0


def test_the_most_work_of_a_call(P):
    """Units of work are counted in 31 bits: 31 streams of the widest tables fit, 32 do not."""
    import ctypes as C

    from paper_2609_02780_amd import _lib as L
    fake, h = 0x7F0000000000, C.c_void_p()
    d = L.CacheDesc(1, 28, 4, 128, 10, 600)
    assert L.lib().ss_cache_create(C.byref(d), fake, 1 << 60, C.byref(h)) == 0
    rows = L.Rows(fake, 128 * 512, 128)
    out = L.Rows(fake + (1 << 30), 128 * 512, 128)

    def attend(streams, width, ws=fake + (1 << 31)):
        s = L.CacheStreams(fake, fake, fake, streams, width)
        return L.lib().ss_cache_attend(h, C.byref(s), 0, streams, None, C.byref(rows), 0, None, None, ws, 0, None,
                                       C.byref(out), None)

    # (a workspace of 0 bytes: a call that could be planned is refused for that, and nothing runs)
    assert attend(31, 2 ** 26 - 2) == L.SS_ERR_WORKSPACE
    assert attend(32, 2 ** 26 - 2) == attend(512, 2 ** 26 - 2) == L.SS_ERR_UNSUPPORTED
    for streams in (33, 100, 512):
        widest = (2 ** 31 - 1) // streams - 2
        assert attend(streams, widest) == L.SS_ERR_WORKSPACE
        assert attend(streams, widest + 1) == L.SS_ERR_UNSUPPORTED
    assert L.lib().ss_cache_destroy(h) == 0
