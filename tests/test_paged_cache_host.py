"""Rotary positions and the paged cache on the host: frequencies, sizes, and the calls that
are refused before anything is enqueued.  No GPU."""
import ctypes as C
import math

import numpy as np
import pytest

import paged_ref as R

FAKE = 0x7F0000000000     # 256-byte aligned stand-in address, never dereferenced here


@pytest.fixture(scope="module")
def L():
    import os

    from paper_2609_02780_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_02780_amd.build import build_library
        build_library()
    return _lib


def freqs(L, dims=64, base=10000.0, factor=1.0, original=0.0, fast=32.0, slow=1.0):
    out, gain = (C.c_double * 512)(), C.c_float(-1.0)
    st = L.lib().ss_rotary_freqs(dims, base, factor, original, fast, slow, out, C.byref(gain))
    return st, np.array(out[:max(0, dims) // 2]), gain.value


@pytest.mark.parametrize("kw", [{}, {"dims": 2}, {"dims": 126, "base": 5e5}, {"factor": 4.0}, {"factor": 1.0, "original": 4096.0},
                                {"factor": 8.0, "original": 4096.0}, {"factor": 2.5, "original": 32768.0, "fast": 16.0, "slow": 2.0}])
def test_frequencies(L, kw):
    st, got, gain = freqs(L, **kw)
    assert st == 0
    want, g = R.frequencies(kw.get("dims", 64), *(kw.get(k, v) for k, v in (
        ("base", 10000.0), ("factor", 1.0), ("original", 0.0), ("fast", 32.0), ("slow", 1.0))))
    np.testing.assert_allclose(got * 2 * math.pi, want, rtol=1e-14)
    assert gain == pytest.approx(g, rel=1e-7)


def test_scaling_by_parts_at_its_ends(L):
    """Frequencies with many turns over the original length stay, those with few are divided."""
    _, plain, _ = freqs(L, dims=128)
    _, parts, _ = freqs(L, dims=128, factor=4.0, original=4096.0)
    turns = plain * 4096.0
    assert (parts[turns >= 32] == plain[turns >= 32]).all() and (turns >= 32).sum() > 5
    np.testing.assert_allclose(parts[turns <= 1], plain[turns <= 1] / 4, rtol=1e-14)
    assert (turns <= 1).sum() > 5 and (np.diff(parts) < 0).all()


@pytest.mark.parametrize("kw", [{"dims": 0}, {"dims": 7}, {"dims": -2}, {"dims": 1026}, {"base": 1.0}, {"base": math.nan},
                                {"base": math.inf}, {"factor": 0.5}, {"factor": math.nan}, {"factor": 2.0 ** 21},
                                {"original": -1.0}, {"original": math.inf}, {"fast": 1.0, "slow": 1.0}, {"slow": -1.0}])
def test_frequencies_refused(L, kw):
    assert freqs(L, **kw)[0] == L.SS_ERR_INVALID_ARGUMENT


def desc(L, **kw):
    d = dict(n_layers=2, n_q_heads=28, n_kv_heads=4, head_dim=128, n_pages=10, n_slots=3)
    d.update(kw)
    return L.CacheDesc(**d)


def create(L, **kw):
    d, h = desc(L, **kw), C.c_void_p()
    assert L.lib().ss_cache_create(C.byref(d), FAKE, L.lib().ss_cache_required_bytes(C.byref(d)), C.byref(h)) == 0
    return h


def test_sizes_and_creation(L):
    lib = L.lib()
    n = lib.ss_cache_required_bytes(C.byref(desc(L)))
    page, slot = 2 * 4 * (32 * 128 + 4), 2 * 2 * 4 * 32 * 128 * 2
    assert 2 * (10 * page + 3 * slot) <= n <= 2 * (10 * page + 3 * slot) + 6 * 256 and n % 256 == 0
    # offsets that pass 32 bits
    big = lib.ss_cache_required_bytes(C.byref(desc(L, n_layers=1024, n_pages=2 ** 31 - 1)))
    assert big > 1024 * (2 ** 31 - 1) * page
    for bad in (dict(head_dim=96), dict(n_q_heads=27), dict(n_q_heads=68), dict(n_kv_heads=0), dict(n_q_heads=0),
                dict(n_kv_heads=16, n_q_heads=16), dict(n_layers=0), dict(n_layers=1025), dict(n_pages=0),
                dict(n_pages=2 ** 31), dict(n_slots=0), dict(n_slots=2 ** 20 + 1)):
        assert lib.ss_cache_required_bytes(C.byref(desc(L, **bad))) == 0, bad
    d, h = desc(L), C.c_void_p()
    assert lib.ss_cache_create(C.byref(d), None, n, C.byref(h)) == L.SS_ERR_INVALID_ARGUMENT
    assert lib.ss_cache_create(C.byref(d), FAKE + 128, n, C.byref(h)) == L.SS_ERR_INVALID_ARGUMENT
    assert lib.ss_cache_create(C.byref(d), FAKE, n - 1, C.byref(h)) == L.SS_ERR_CAPACITY
    assert lib.ss_cache_create(C.byref(d), FAKE, n, None) == L.SS_ERR_INVALID_ARGUMENT
    assert lib.ss_cache_destroy(None) == L.SS_ERR_INVALID_ARGUMENT
    assert lib.ss_cache_destroy(create(L)) == 0


def rows(L, heads=4, tokens=6, at=FAKE, hs=None, ts=None, d=128):
    return L.Rows(at, tokens * d if hs is None else hs, d if ts is None else ts)


def streams(L, n=3, width=5, **kw):
    a = dict(tables=FAKE, lengths=FAKE, slots=FAKE)
    a.update(kw)
    return L.CacheStreams(a["tables"], a["lengths"], a["slots"], n, width)


def ints(*v):
    return (C.c_int32 * len(v))(*v)


def test_rotation_refused(L):
    lib = L.lib()
    r, x, y = L.Rotary(FAKE, 64, 0, 1.0), rows(L), rows(L, at=FAKE + 65536)

    def call(rotary=r, heads=4, tokens=6, d=128, x=x, pos=FAKE, out=y):
        ref = lambda v: C.byref(v) if v is not None else None     # noqa: E731
        return lib.ss_rotate(ref(rotary), heads, tokens, d, ref(x), pos, 0, ref(out), None)

    assert call(rotary=None) == call(rotary=L.Rotary(None, 64, 0, 1.0)) == L.SS_ERR_INVALID_ARGUMENT
    for dims in (0, 1, 65, 130):
        assert call(rotary=L.Rotary(FAKE, dims, 0, 1.0)) == L.SS_ERR_INVALID_ARGUMENT
    assert call(rotary=L.Rotary(FAKE, 128, 0, 1.0), d=64) == L.SS_ERR_INVALID_ARGUMENT
    assert call(rotary=L.Rotary(FAKE, 64, 0, math.nan)) == L.SS_ERR_INVALID_ARGUMENT
    assert call(d=96) == call(heads=0) == call(heads=4097) == call(tokens=65537) == L.SS_ERR_UNSUPPORTED
    assert call(tokens=0) == call(x=None) == call(out=None) == call(pos=None) == call(pos=FAKE + 4) == L.SS_ERR_INVALID_ARGUMENT
    assert call(x=rows(L, at=FAKE + 8)) == call(x=rows(L, hs=12)) == call(x=rows(L, ts=-128)) == L.SS_ERR_INVALID_ARGUMENT
    # rows of the output that overlap, or lie on x with other strides
    for bad in (rows(L, at=FAKE + 65536, ts=64), rows(L, at=FAKE + 65536, hs=0), rows(L, at=FAKE + 65536, hs=128),
                rows(L, ts=256, hs=6 * 256)):
        assert call(out=bad) == L.SS_ERR_INVALID_ARGUMENT, (bad.head_stride, bad.token_stride)
    assert b"strides" in lib.ss_last_error()


def test_append_and_attention_refused(L):
    lib, h = L.lib(), create(L)
    k, q, o = rows(L), rows(L, 28, at=FAKE + (1 << 20)), rows(L, 28, at=FAKE + (1 << 21))
    ref = lambda v: C.byref(v) if v is not None else None         # noqa: E731

    def append(cache=h, s=streams(L), layer=1, tokens=6, n=None, k=k, v=k, rot=L.Rotary(FAKE, 64, 0, 1.0), pos=None, q=q, qo=o):
        return lib.ss_cache_append(cache, ref(s), layer, tokens, n, ref(k), ref(v), ref(rot), pos, ref(q), ref(qo), None)

    def attend(cache=h, s=streams(L), layer=1, tokens=6, n=None, q=q, window=0, po=None, pl=None, ws=FAKE, nbytes=1 << 30,
               out=o, lse=FAKE):
        return lib.ss_cache_attend(cache, ref(s), layer, tokens, n, ref(q), window, ref(po), pl, ws, nbytes, None, ref(out), lse)

    bad = L.SS_ERR_INVALID_ARGUMENT
    for call in (append, attend):
        assert call(cache=None) == call(s=None) == call(layer=-1) == call(layer=2) == call(tokens=0) == bad
        assert call(tokens=7) == bad and b"same number" in lib.ss_last_error()
        assert call(n=ints(1, 2, 4)) == call(n=ints(-1, 3, 4)) == bad
        assert call(tokens=65539, n=ints(65539, 0, 0)) == L.SS_ERR_UNSUPPORTED
        assert call(s=streams(L, n=0)) == call(s=streams(L, n=513)) == L.SS_ERR_UNSUPPORTED
        assert call(s=streams(L, width=0)) == call(s=streams(L, width=2 ** 26 - 1)) == L.SS_ERR_UNSUPPORTED
        for name in ("tables", "lengths", "slots"):
            assert call(s=streams(L, **{name: None})) == call(s=streams(L, **{name: FAKE + 2})) == bad
    assert append(k=None) == append(v=None) == append(k=rows(L, at=FAKE + 4)) == append(v=rows(L, hs=4)) == bad
    assert append(rot=L.Rotary(FAKE, 130, 0, 1.0)) == append(rot=None, pos=FAKE) == append(pos=FAKE + 4) == bad
    assert append(q=None) == append(qo=None) == append(qo=rows(L, 28, at=o.data, hs=0)) == append(qo=k) == bad
    assert append(qo=rows(L, 28, at=q.data, hs=128, ts=28 * 128)) == bad
    assert attend(q=None) == attend(out=None) == attend(out=q) == attend(out=rows(L, 28, at=o.data, ts=0)) == bad
    assert attend(window=-1) == attend(window=2 ** 30 + 1) == attend(lse=FAKE + 2) == bad
    assert attend(po=k) == attend(pl=FAKE) == attend(po=o, pl=FAKE) == attend(po=q, pl=FAKE, lse=FAKE) == bad
    assert attend(ws=None) == attend(ws=FAKE + 64) == L.SS_ERR_WORKSPACE
    assert attend(s=streams(L, width=5000), nbytes=1024) == L.SS_ERR_WORKSPACE
    # units of work are counted in 31 bits
    wide = dict(s=streams(L, n=512, width=2 ** 26 - 2), tokens=512, q=rows(L, 28, 512), out=rows(L, 28, 512, at=o.data))
    assert attend(**wide) in (L.SS_ERR_UNSUPPORTED, L.SS_ERR_WORKSPACE)
    need = lib.ss_cache_attend_workspace_bytes
    s = streams(L)
    assert need(h, C.byref(s), 6, None, 0) == 256 and need(h, C.byref(s), 7, None, 0) == 0
    assert lib.ss_cache_destroy(h) == 0


def test_workspace_is_the_least_where_units_are_short(L):
    """A short table takes a block a unit, which writes no workspace; a long one is cut into shares."""
    lib, h = L.lib(), create(L)
    need = lambda width, tokens, window=0, n=1: lib.ss_cache_attend_workspace_bytes(   # noqa: E731
        h, C.byref(streams(L, n=n, width=width)), tokens, None, window)
    assert need(30, 1) == 256 and need(20000, 1) > 256
    assert need(20000, 1, window=500) == 256
    assert need(200, 64) > 256 and need(4, 64) == 256
    # a part of 7 columns and 128 dimensions for each of at most 1,024 slots, and its statistics
    assert need(20000, 1) <= 1024 * 7 * (128 + 3) * 4 + 4096
    assert lib.ss_cache_destroy(h) == 0


def test_binding_refuses_before_the_library(L):
    """Host tensors and wrong shapes name the argument."""
    import torch

    from paper_2609_02780_amd import paged
    dev = torch.device("cuda", 0)
    x = torch.zeros(4, 6, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="keys lives on cpu"):
        paged._rows(x, (4, 6, 128), dev, "keys")
    with pytest.raises(ValueError, match="keys must be a bfloat16"):
        paged._rows(x.float(), (4, 6, 128), dev, "keys")
    with pytest.raises(ValueError, match=r"keys has shape \(4, 6, 128\)"):
        paged._rows(x, (4, 7, 128), dev, "keys")
    with pytest.raises(ValueError, match="side by side"):
        paged._rows(x.transpose(1, 2), (4, 128, 6), x.device, "keys")
    with pytest.raises(ValueError, match="lengths must be a contiguous torch.int32"):
        paged._ints(torch.zeros(3), (3,), torch.int32, dev, "lengths")
    with pytest.raises(ValueError, match="lengths lives on cpu"):
        paged._ints(torch.zeros(3, dtype=torch.int32), (3,), torch.int32, dev, "lengths")
    r = paged._rows(x[:, :1], (4, 1, 128), x.device, "keys")
    assert (r.head_stride, r.token_stride) == (6 * 128, 0)
