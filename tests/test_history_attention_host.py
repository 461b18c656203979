"""Host-side refusals of the value cache, attention over the history and eviction:
every call here fails validation (or is a host query) and enqueues nothing."""
import ctypes as C
import math
import os

import numpy as np
import pytest

import history_ref as R

FAKE = 0x7F0000000000     # 256-byte aligned stand-in address, never dereferenced here


@pytest.fixture(scope="module")
def L():
    from paper_2609_02780_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_02780_amd.build import build_library
        build_library()
    return _lib


def make(L, values=True, at=FAKE, **kw):
    d = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_frames=10, max_rows=100, n_recent=2)
    d.update(kw)
    desc = L.IndexDesc(**d)
    h = C.c_void_p()
    assert L.lib().ss_index_create(C.byref(desc), at, L.lib().ss_index_required_bytes(C.byref(desc)), C.byref(h)) == 0
    if values:
        n = L.lib().ss_values_required_bytes(C.byref(desc))
        assert L.lib().ss_index_attach_values(h, at + (1 << 32), n) == 0
    return h


class Call:
    """One attend call's arguments, changed by name."""

    def __init__(self, L, idx, **kw):
        S = len(idx)
        self.L, self.S = L, S
        self.idx = (C.c_void_p * S)(*idx)
        self.q = (C.c_void_p * S)(*[FAKE] * S)
        self.n_q = (C.c_int32 * S)(*[3] * S)
        self.prm = L.AttendParams(1, 0.0, None, None, None, 0)
        self.ok_k = (C.c_void_p * S)(*[FAKE] * S)
        self.ok_v = (C.c_void_p * S)(*[FAKE] * S)
        self.n_own = (C.c_int32 * S)(*[5] * S)
        self.cap = (C.c_int32 * S)(*[8] * S)
        self.par = (C.c_void_p * S)(*[None] * S)
        self.own = L.OwnTokens(C.cast(self.ok_k, C.c_void_p), C.cast(self.ok_v, C.c_void_p),
                               C.cast(self.n_own, C.c_void_p), C.cast(self.cap, C.c_void_p),
                               C.cast(self.par, C.c_void_p))
        self.out = (C.c_void_p * S)(*[FAKE + 4096 + 256 * s for s in range(S)])
        self.lse = (C.c_void_p * S)(*[FAKE + 8192 + 256 * s for s in range(S)])
        self.ws, self.ws_bytes, self.decay = FAKE, 0, 1.0     # a workspace of 0 bytes: the last check fails
        for k, v in kw.items():
            setattr(self, k, v)

    def attend(self):
        return self.L.lib().ss_attend(self.idx, self.S, self.q, self.n_q, C.byref(self.own) if self.own else None,
                                      C.byref(self.prm), self.ws, self.ws_bytes, None, self.out, self.lse)

    def accumulate(self):
        return self.L.lib().ss_attend_accumulate(self.idx, self.S, self.q, self.n_q, self.lse, C.byref(self.prm),
                                                 self.decay, self.ws, self.ws_bytes, None)

    def bytes(self):
        return self.L.lib().ss_attend_workspace_bytes(self.idx, self.S, self.n_q,
                                                      C.byref(self.own) if self.own else None, C.byref(self.prm))


def err(L):
    return L.lib().ss_last_error().decode()


def test_values_arena(L):
    d = L.IndexDesc(2, 8, 2, 64, 10, 100, 0)
    n = L.lib().ss_values_required_bytes(C.byref(d))
    assert n == 2 * 2 * 100 * 64 * 2 + (2 * 2 * 100 * 4 + 255) // 256 * 256
    assert L.lib().ss_values_required_bytes(C.byref(L.IndexDesc(2, 8, 2, 96, 10, 100, 0))) == 0
    h = make(L, values=False)
    f = L.lib().ss_index_attach_values
    assert f(None, FAKE, n) == L.SS_ERR_INVALID_ARGUMENT
    assert f(h, None, n) == L.SS_ERR_INVALID_ARGUMENT
    assert f(h, FAKE + 64, n) == L.SS_ERR_INVALID_ARGUMENT
    assert f(h, FAKE, n - 1) == L.SS_ERR_CAPACITY and "needed" in err(L)
    assert f(h, FAKE, n) == 0
    assert f(h, FAKE, n) == L.SS_ERR_INVALID_ARGUMENT and "already" in err(L)
    L.lib().ss_index_destroy(h)


def test_append_needs_the_right_entry(L):
    kv, plain = make(L), make(L, values=False)
    p = L.ptr_array([FAKE, FAKE])
    bad = L.ptr_array([FAKE, FAKE + 2])
    null = L.ptr_array([FAKE, None])
    f = L.lib()
    assert f.ss_index_append(kv, p, 1, 4, None, None, None) == L.SS_ERR_INVALID_ARGUMENT and "append_kv" in err(L)
    assert f.ss_index_append_kv(plain, p, p, 1, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(None, p, p, 1, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(kv, p, None, 1, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(kv, p, bad, 1, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(kv, p, null, 1, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(kv, null, p, 1, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(kv, p, p, 0, 4, None, None) == L.SS_ERR_INVALID_ARGUMENT
    assert f.ss_index_append_kv(kv, p, p, 11, 4, None, None) == L.SS_ERR_CAPACITY
    assert f.ss_index_append_kv(kv, p, p, 2, 51, None, None) == L.SS_ERR_CAPACITY
    for h in (kv, plain):
        f.ss_index_destroy(h)


def test_attend_refusals(L):
    kv, plain, other = make(L), make(L, values=False), make(L, n_q_heads=4)
    inv, uns = L.SS_ERR_INVALID_ARGUMENT, L.SS_ERR_UNSUPPORTED

    def status(change=None, idx=None, fn="attend"):
        c = Call(L, idx or [kv.value])
        if change:
            change(c)
        return getattr(c, fn)()

    assert status() == L.SS_ERR_WORKSPACE                       # everything else holds
    assert status(fn="accumulate") == L.SS_ERR_WORKSPACE

    def put(name, i, v):
        return lambda c: getattr(c, name).__setitem__(i, v)

    def field(name, v):
        return lambda c: setattr(c.prm, name, v)

    for fn in ("attend", "accumulate"):
        assert status(idx=[plain.value], fn=fn) == inv and "values" in err(L)
        assert status(idx=[kv.value, other.value], fn=fn) == inv and "shape" in err(L)
        assert status(put("idx", 0, None), fn=fn) == inv
        for n in (0, -1, 4097):
            assert status(put("n_q", 0, n), fn=fn) == inv
        for l in (-1, 2):
            assert status(field("layer", l), fn=fn) == inv
        for c in (-1.0, math.inf, math.nan):
            assert status(field("softcap", c), fn=fn) == inv
        for c in (1e-4, 1e7):
            assert status(field("softcap", c), fn=fn) == uns
        assert status(field("n_listed", 4), fn=fn) == inv
        assert status(field("kinds", FAKE), fn=fn) == inv
        assert status(field("slopes", FAKE + 2), fn=fn) == inv

        def listed(n, frames=FAKE, kinds=None):
            def f(c):
                c.prm.frames, c.prm.n_listed, c.prm.kinds = frames, n, kinds
            return f
        assert status(listed(0), fn=fn) == uns
        assert status(listed(4097), fn=fn) == uns
        assert status(listed(4, FAKE + 4), fn=fn) == inv
        assert status(listed(4, FAKE, FAKE + 2), fn=fn) == inv
        assert status(listed(4096, FAKE, FAKE), fn=fn) == L.SS_ERR_WORKSPACE
        assert status(put("q", 0, None), fn=fn) == inv
        assert status(put("q", 0, FAKE + 8), fn=fn) == inv
        assert status(put("lse", 0, FAKE + 2), fn=fn) == inv
        assert status(put("lse", 0, None), fn=fn) == inv
        assert status(lambda c: setattr(c, "ws", FAKE + 16), fn=fn) == L.SS_ERR_WORKSPACE
        assert status(lambda c: setattr(c, "ws", None), fn=fn) == L.SS_ERR_WORKSPACE
    assert status(put("out", 0, None)) == inv
    assert status(put("out", 0, FAKE + 4)) == inv
    assert status(put("out", 0, FAKE)) == inv and "queries" in err(L)
    for name in ("out", "lse"):
        assert status(lambda c: getattr(c, name).__setitem__(1, getattr(c, name)[0]), idx=[kv.value] * 2) == inv
        assert "one output" in err(L)
    for n in (1, 2, -1, (1 << 20) + 1):
        assert status(put("n_own", 0, n)) == inv
    assert status(put("n_own", 0, 0)) == L.SS_ERR_WORKSPACE
    for n in (4, (1 << 20) + 1):
        assert status(put("cap", 0, n)) == inv
    assert status(put("ok_k", 0, None)) == inv
    assert status(put("ok_v", 0, FAKE + 8)) == inv
    assert status(put("par", 0, FAKE + 2)) == inv

    def tree(nq, nown):
        def f(c):
            c.par[0], c.n_q[0], c.n_own[0], c.cap[0] = FAKE, nq, nown, max(nown, 8)
        return f
    assert status(tree(3, 0)) == inv
    assert status(tree(513, 600)) == uns
    assert status(tree(512, 600)) == L.SS_ERR_WORKSPACE
    for d in (-0.1, 1.1, math.nan):
        assert status(lambda c: setattr(c, "decay", d), fn="accumulate") == inv
    assert status(idx=[kv.value, kv.value], fn="accumulate") == inv and "one index" in err(L)
    assert status(idx=[kv.value, kv.value]) == L.SS_ERR_WORKSPACE
    c = Call(L, [kv.value])
    assert c.bytes() > 0 and c.bytes() % 256 == 0
    c.n_q[0] = 0
    assert c.bytes() == 0
    for h in (kv, plain, other):
        L.lib().ss_index_destroy(h)


def test_workspace_of_every_shape(L):
    """The planner ends, and asks for whole 256-byte pieces, over the documented sizes."""
    rng = np.random.default_rng(1)
    for n_q_heads, n_kv, d in ((1, 1, 64), (16, 1, 128), (16, 16, 64), (28, 4, 128), (8, 8, 128)):
        h = make(L, n_q_heads=n_q_heads, n_kv_heads=n_kv, head_dim=d)
        for _ in range(60):
            S = int(rng.choice([1, 2, 16, 17, 33]))
            c = Call(L, [h.value] * S)
            for s in range(S):
                c.n_q[s] = int(rng.choice([1, 2, 31, 64, 1000, 4096, rng.integers(1, 4097)]))
                c.n_own[s] = int(rng.choice([0, c.n_q[s], 1 << 20, rng.integers(c.n_q[s], 1 << 20)]))
                c.cap[s] = 1 << 20
            if rng.random() < 0.5:
                c.prm.frames, c.prm.n_listed = FAKE, int(rng.integers(1, 4097))
            n = c.bytes()
            assert n >= 256 and n % 256 == 0
            m = L.lib().ss_attend_accumulate_workspace_bytes(c.idx, S, c.n_q, C.byref(c.prm))
            assert m >= 256 and m % 256 == 0
        L.lib().ss_index_destroy(h)


def test_evict_refusals(L):
    a, plain, other = make(L), make(L, values=False), make(L, head_dim=128)
    b = make(L, at=FAKE + (1 << 34))
    overlap = make(L, at=FAKE + (1 << 32))      # its index arena lies in a's value arena
    f, inv = L.lib().ss_index_evict, L.SS_ERR_INVALID_ARGUMENT
    assert f(None, b, 0, 4, None) == inv and f(a, None, 0, 4, None) == inv
    assert f(a, a, 0, 4, None) == inv
    assert f(a, plain, 0, 4, None) == inv and f(plain, b, 0, 4, None) == inv
    assert f(a, other, 0, 4, None) == inv
    assert f(a, overlap, 0, 4, None) == inv and "overlap" in err(L)
    assert f(overlap, a, 0, 4, None) == inv
    assert f(a, b, 0, 0, None) == inv
    assert f(a, b, 1, 4, None) == inv and f(a, b, -1, 4, None) == inv
    for h in (a, b, plain, other, overlap):
        L.lib().ss_index_destroy(h)


def test_reference_by_hand():
    """The 64-bit forms on cases worked by hand."""
    q = np.zeros((1, 1, 4))
    k = np.ones((1, 3, 4))
    v = np.array([[[0.0, 3, 0, 0], [3, 0, 0, 0], [0, 0, 3, 6]]])
    out, lse, _, _ = R.attend(q, k, v, np.ones((1, 3), dtype=bool), 1)
    assert np.allclose(out[0, 0], [1, 1, 1, 2]) and np.allclose(lse, math.log(3))
    # a bias of ln 2 a frame halves the weight with each frame: 1/2, 1/4, 1/8
    out, lse, _, _ = R.attend(q, k, v, np.ones((1, 3), dtype=bool), 1, slopes=np.array([math.log(2)]),
                              age=np.array([3.0, 2, 1]))
    assert np.allclose(out[0, 0], [6 / 7, 3 / 7, 12 / 7, 24 / 7]) and np.allclose(lse, math.log(7 / 8))
    w, _ = R.weights(q, k, lse, 1, slopes=np.array([math.log(2)]), age=np.array([3.0, 2, 1]))
    assert np.allclose(w, [[1 / 7, 2 / 7, 4 / 7]])
    q = np.full((1, 1, 4), 50.0)                       # scores of 100, capped at 2
    out, lse, _, _ = R.attend(q, k, v, np.array([[True, False, False]]), 1, softcap=2.0)
    assert np.allclose(out[0, 0], v[0, 0]) and np.allclose(lse, 2.0)
    out, lse, _, _ = R.attend(q, k, v, np.zeros((1, 3), dtype=bool), 1)
    assert not out.any() and np.isneginf(lse).all()
    assert R.tree_mask([-1, 0, 0, 1, 9], 6).tolist() == [
        [True, True, False, False, False, False], [True, True, True, False, False, False],
        [True, True, False, True, False, False], [True, True, True, False, True, False],
        [True, False, False, False, False, True]]
    assert R.causal(2, 3).tolist() == [[True, True, False], [True, True, True]]
    assert R.kept_rows(np.array([1, 3, 3, 0, 5.0, 4]), [4, 2], 1, 2).tolist() == [1, 2, 4, 5]
    assert R.kept_rows(np.array([1, 3, 3, 3.0]), [4], 1, 2).tolist() == [1, 2]
