"""Rotary positions, a paged cache of keys and values in 8 bits, and attention over it.

The binding's rules are those of ``index.py``: argument marshalling only, tensors on the
current HIP device, bfloat16 rows.  Rows of several heads are tensors ``[heads][tokens][d]``
with any strides of heads and tokens that are multiples of 16 bytes (a projection's
``[tokens][heads][d]`` may be given as its transposed view).
"""
from __future__ import annotations

import ctypes as C

import torch

from . import _lib as L
from .index import _on_current, _raw_stream, _returned_from, _stream_handle, _used_on

_BF16 = torch.bfloat16


def _rows(t, shape: tuple, device, what: str) -> L.Rows:
    """A tensor ``[heads][tokens][d]`` of this shape as the C ABI takes it (which checks alignment and strides)."""
    if not isinstance(t, torch.Tensor) or t.dtype is not _BF16:
        raise ValueError(f"{what} must be a bfloat16 tensor")
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {shape}")
    if t.device != device:
        raise ValueError(f"{what} lives on {t.device}, expected {device}")
    hs, ts, one = t.stride()
    if one != 1:
        raise ValueError(f"the elements of a row of {what} must lie side by side")
    # a dimension of one row has any stride
    return L.Rows(t.data_ptr(), hs if shape[0] > 1 else 0, ts if shape[1] > 1 else 0)


def _like(stream, x, r: L.Rows):
    """A new tensor laid out as ``x``, whose rows are ``r``, and its rows."""
    out = torch.empty_like(x) if stream is None else _new(stream, torch.empty_like, x)
    if out.stride() == x.stride():
        return out, L.Rows(out.data_ptr(), r.head_stride, r.token_stride)
    return out, _rows(out, out.shape, out.device, "out")


def _new(stream, f, *args, **kw):
    """``f``'s new tensor, in memory of the stream that fills it."""
    if stream is None:
        return f(*args, **kw)
    with torch.cuda.stream(stream):
        return f(*args, **kw)


def _launch_stream(stream, device) -> int:
    """The handle of the stream that a call on the current device runs on."""
    if stream is None and _raw_stream is not None:
        return _raw_stream(device.index)
    return _stream_handle(stream)


def _ints(t, shape, dtype, device, what: str) -> int:
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} tensor {list(shape)}")
    if t.device != device:
        raise ValueError(f"{what} lives on {t.device}, expected {device}")
    return t.data_ptr()


class Rotary:
    """Rotary positions of the first ``dims`` elements of a head: pairs ``(i, i + dims / 2)``, or
    neighbours with ``interleaved``, turned by ``position * base ** (-2 i / dims)``.

    For contexts ``factor`` times as long: all frequencies divided by it, or with
    ``original`` (the length that the model was trained at) by parts, where those with
    ``fast`` turns and more over that length stay, those with ``slow`` and fewer are divided
    and the ones between are mixed; the result is then scaled by ``1 + 0.1 ln(factor)``
    (``gain``: by that instead).

    Frequencies of any other rule are written in place, ``rotary.freqs.copy_(...)``: fp64
    ``[dims / 2]`` on the device, in turns a position.  Calls that are captured read them there too.
    """

    def __init__(self, dims: int, base: float = 10000.0, interleaved: bool = False, factor: float = 1.0,
                 original: float = 0.0, fast: float = 32.0, slow: float = 1.0, gain: float | None = None, device=None):
        freqs, g = torch.empty(max(dims, 2) // 2, dtype=torch.float64), C.c_float()
        L.check(L.lib().ss_rotary_freqs(dims, base, factor, original, fast, slow, freqs.data_ptr(), C.byref(g)))
        dev = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
        self._freqs = freqs.to(dev)
        self._device, self._lib = self._freqs.device, L.lib()
        self._c = L.Rotary(self._freqs.data_ptr(), dims, int(bool(interleaved)), float(g.value if gain is None else gain))
        self._ref = C.byref(self._c)

    # What a call uses is `_c`, so nothing here is exchanged.  (What writes in place, as `rotary.freqs /= 2`, assigns
    # the tensor that is there.)
    @property
    def freqs(self) -> torch.Tensor:
        return self._freqs

    @freqs.setter
    def freqs(self, t) -> None:
        if t is not self._freqs:
            raise ValueError("freqs of a rotation are written in place")

    @property
    def dims(self) -> int:
        return self._c.dims

    @property
    def interleaved(self) -> bool:
        return bool(self._c.interleaved)

    @property
    def gain(self) -> float:
        return self._c.gain

    def __call__(self, x, positions, transposed: bool = False, out=None, stream=None):
        """``x``: ``[heads][tokens][d]`` bfloat16; ``positions``: int64 ``[tokens]``.  Returns ``out``
        (``x`` itself may be given), by default a new tensor laid out as ``x``.  ``transposed`` is
        the gradient of the rotation, and undoes it when ``gain`` is 1."""
        if not isinstance(x, torch.Tensor) or x.dim() != 3:
            raise ValueError("x must be [heads][tokens][d]")
        _on_current(self._device, "the frequencies live")
        shape = x.shape
        H, N, d = shape
        dev = self._device
        src = _rows(x, shape, dev, "x")
        at = _ints(positions, (N,), torch.int64, dev, "positions")
        fresh = out is None
        if fresh:
            out, dst = _like(stream, x, src)
        else:
            dst = _rows(out, shape, dev, "out")
        L.check(self._lib.ss_rotate(self._ref, H, N, d, C.byref(src), at, transposed, C.byref(dst),
                                    _launch_stream(stream, dev)))
        if stream is not None:
            _used_on(stream, x, positions, self._freqs)
            if fresh:
                _returned_from(stream, out)
            else:
                _used_on(stream, out)
        return out


class PagedCache:
    """Keys and values of any number of layers and streams in 8 bits: pages of 32 tokens,
    e4m3 with a scale for each page and KV head, in a device arena owned by this object.

    A page holds its block at every layer; which pages are a stream's is the caller's to say
    (:class:`PagedBatch`).  A stream's tokens behind its last full block stay bfloat16 in one
    of ``n_slots`` slots.

    The views below hold one tensor a layer, which may be read and written.  ``keys[l]`` is
    ``[n_pages][H_kv][32][d/16][16]`` and ``values[l]`` ``[n_pages][H_kv][2][2][2][4][d/32][32]``, both
    ``[...][32][d]`` with tokens and dimensions cut as memory has them (``reshape`` to that copies);
    ``key_scales[l]`` and ``value_scales[l]`` fp32 ``[n_pages][H_kv]``; ``open_keys[l]`` and
    ``open_values[l]`` bfloat16 ``[n_slots][2][H_kv]`` and then as the pages, block ``b`` in half ``b & 1``.
    """

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, n_pages: int, n_slots: int,
                 device=None):
        self.desc = L.CacheDesc(n_layers, n_q_heads, n_kv_heads, head_dim, n_pages, n_slots)
        nbytes = L.lib().ss_cache_required_bytes(C.byref(self.desc))
        if nbytes == 0:
            raise L.SSError(L.SS_ERR_INVALID_ARGUMENT, L.lib().ss_last_error().decode())
        dev = torch.device(device) if device is not None else torch.device("cuda", torch.cuda.current_device())
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        self._h = C.c_void_p()
        L.check(L.lib().ss_cache_create(C.byref(self.desc), self.arena.data_ptr(), nbytes, C.byref(self._h)))
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        self.n_pages, self.n_slots = n_pages, n_slots
        at = 0

        def part(dtype, *shape):
            nonlocal at
            n = dtype.itemsize
            for x in shape:
                n *= x
            t = self.arena[at:at + n].view(dtype).view(shape)
            at = (at + n + 255) // 256 * 256
            return t

        pages, slots, d = (n_layers, n_pages, n_kv_heads), (n_layers, n_slots, 2, n_kv_heads), head_dim
        key, value = (d // 16, 32, 16), (d // 32, 2, 32, 2, 2, 4)

        def by_token(k, v):
            """[32][d/16][16] of [d/16][32][16], and [2][2][2][4][d/32][32] of the values' order."""
            n = k.dim() - 3
            lead = list(range(n))
            return (k.permute(*lead, n + 1, n, n + 2), v.permute(*lead, n + 4, n + 3, n + 1, n + 5, n, n + 2))

        k, v = part(torch.float8_e4m3fn, *pages, *key), part(torch.float8_e4m3fn, *pages, *value)
        self.keys, self.values = (t.unbind(0) for t in by_token(k, v))
        self.key_scales, self.value_scales = part(torch.float32, *pages).unbind(0), part(torch.float32, *pages).unbind(0)
        k, v = part(_BF16, *slots, *key), part(_BF16, *slots, *value)
        self.open_keys, self.open_values = (t.unbind(0) for t in by_token(k, v))

    @property
    def handle(self) -> C.c_void_p:
        if self._h is None:
            raise RuntimeError("cache closed")
        return self._h

    def close(self) -> None:
        if getattr(self, "_h", None) is not None:
            L.check(L.lib().ss_cache_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PagedBatch:
    """Streams of a :class:`PagedCache` that are worked on together.

    ``tables`` int32 ``[S][width]``: the page of each of a stream's blocks of 32 tokens;
    ``lengths`` int32 ``[S]``: its tokens, those of the next call among them; ``slots`` int32
    ``[S]``: where its open block lies.  The tensors stay the caller's, who writes them between
    calls (a captured call follows them), as in::

        batch.lengths += 1
        for layer in range(n_layers):
            q = batch.append(layer, keys, values, rotary=rotary, queries=queries)
            out, lse = batch.attend(layer, q)

    Nothing is kept between calls but these three, so calls on different streams or in different
    captured graphs share nothing but the cache.  A caller that gives a ``stream`` orders it
    behind its inputs, and what reads the outputs behind it.
    """

    def __init__(self, cache: PagedCache, tables: torch.Tensor, lengths: torch.Tensor, slots: torch.Tensor):
        dev = cache.arena.device
        if not isinstance(tables, torch.Tensor) or tables.dim() != 2:
            raise ValueError("tables must be [n_streams][width]")
        S, width = tables.shape
        self._cache, self._tables, self._lengths, self._slots = cache, tables, lengths, slots
        self._device, self._lib, self._S = dev, L.lib(), S
        self._c = L.CacheStreams(_ints(tables, (S, width), torch.int32, dev, "tables"),
                                 _ints(lengths, (S,), torch.int32, dev, "lengths"),
                                 _ints(slots, (S,), torch.int32, dev, "slots"), S, width)
        self._ref = C.byref(self._c)
        self._counts_type = C.c_int32 * max(S, 1)
        self._least = torch.empty(256, dtype=torch.uint8, device=dev)
        self._needs, self._fp32 = {}, torch.empty(1, dtype=torch.float32, device=dev)

    # (workspaces and outputs are formed by its heads)
    @property
    def cache(self) -> PagedCache:
        return self._cache

    # (what writes in place, as `batch.lengths += 1`, assigns the tensor that is there)
    @property
    def tables(self) -> torch.Tensor:
        return self._tables

    @tables.setter
    def tables(self, t) -> None:
        self._same(t, self._tables, "tables")

    @property
    def lengths(self) -> torch.Tensor:
        return self._lengths

    @lengths.setter
    def lengths(self, t) -> None:
        self._same(t, self._lengths, "lengths")

    @property
    def slots(self) -> torch.Tensor:
        return self._slots

    @slots.setter
    def slots(self, t) -> None:
        self._same(t, self._slots, "slots")

    @staticmethod
    def _same(t, held, what: str) -> None:
        if t is not held:
            raise ValueError(f"{what} of a batch are written in place; make a new batch for another tensor")

    def _counts(self, n, what: str):
        if n is None:
            return None
        if len(n) != self._S:
            raise ValueError(f"{what} must hold a number for each of {self._S} streams")
        return self._counts_type(*n)

    def append(self, layer: int, keys, values, n_new=None, rotary: Rotary | None = None, positions=None, queries=None,
               queries_out=None, stream=None):
        """Append rows ``[H_kv][tokens][d]``, the streams' one after another: ``n_new[s]`` each (default: the
        same number).  Keys are rotated by ``rotary`` at ``positions`` (int64 ``[tokens]``; default: a token's
        place in its stream).  ``queries`` ``[H_q][tokens][d]`` are rotated alike and returned
        (in ``queries_out``, which may be ``queries``; by default a new tensor laid out as they are)."""
        c, dev = self._cache, self._device
        _on_current(dev, "the cache lives")
        if not isinstance(keys, torch.Tensor) or keys.dim() != 3:
            raise ValueError("keys must be [n_kv_heads][tokens][d]")
        N, d = keys.shape[1], c.head_dim
        shape = (c.n_kv_heads, N, d)
        k = _rows(keys, shape, dev, "keys")
        v = _rows(values, shape, dev, "values")
        rot, at = None, None
        if rotary is not None:
            if rotary._device != dev:
                raise ValueError(f"rotary lives on {rotary._device}, the cache on {dev}")
            rot = rotary._ref
        if positions is not None:
            at = _ints(positions, (N,), torch.int64, dev, "positions")
        q = qo = None
        out = queries_out
        if queries is not None:
            shape = (c.n_q_heads, N, d)
            q = _rows(queries, shape, dev, "queries")
            if out is None:
                out, qo = _like(stream, queries, q)
            else:
                qo = _rows(out, shape, dev, "queries_out")
            q, qo = C.byref(q), C.byref(qo)
        elif out is not None:
            raise ValueError("queries_out without queries")
        L.check(self._lib.ss_cache_append(c.handle, self._ref, layer, N, self._counts(n_new, "n_new"), C.byref(k),
                                          C.byref(v), rot, at, q, qo, _launch_stream(stream, dev)))
        if stream is not None:
            _used_on(stream, c.arena, self.tables, self.lengths, self.slots, keys, values, positions, queries,
                     queries_out, rotary.freqs if rotary is not None else None)
            if out is not None and queries_out is None:
                _returned_from(stream, out)
        return out

    def attend(self, layer: int, queries, n_q=None, window: int = 0, prior=None, stream=None):
        """Attention of the streams' last tokens: ``queries`` ``[H_q][tokens][d]``, ``n_q[s]`` of each stream
        (default: the same number).  Each sees its stream up to itself, with ``window`` the newest
        so many of those tokens.  ``prior``: ``(out, lse)`` of the same queries over other rows, which
        the result is joined with (as :class:`HistoryAttention` returns them; bfloat16 ``[H_q][tokens][d]``
        and fp32 ``[H_q][tokens]``).  Returns ``(out, lse)``, ``out`` laid out as ``queries``."""
        c, dev, lib = self._cache, self._device, self._lib
        _on_current(dev, "the cache lives")
        if not isinstance(queries, torch.Tensor) or queries.dim() != 3:
            raise ValueError("queries must be [n_q_heads][tokens][d]")
        N, d, Hq = queries.shape[1], c.head_dim, c.n_q_heads
        q = _rows(queries, (Hq, N, d), dev, "queries")
        po = pl = None
        if prior is not None:
            po = C.byref(_rows(prior[0], (Hq, N, d), dev, "prior out"))
            pl = _ints(prior[1], (Hq, N), torch.float32, dev, "prior lse")
        n = self._counts(n_q, "n_q")
        # (calls with the same number of queries for every stream, whose size is theirs alone, ask for it once)
        need, like = self._needs.get((N, window), (None, None)) if n is None else (None, None)
        if need is None:
            need = lib.ss_cache_attend_workspace_bytes(c.handle, self._ref, N, n, window)
            if need == 0:
                raise L.SSError(L.SS_ERR_INVALID_ARGUMENT, lib.ss_last_error().decode())
            like = self._fp32.expand(Hq, N)                 # (an empty tensor like it takes less of the host than one by size)
            if n is None:
                if len(self._needs) >= 256:
                    self._needs.clear()
                self._needs[N, window] = need, like
        # a need of 256, the least, is of a call that writes no workspace: those share one
        ws = self._least if need == 256 else _new(stream, torch.empty, need, dtype=torch.uint8, device=dev)
        out, o = _like(stream, queries, q)
        lse = torch.empty_like(like) if stream is None else _new(stream, torch.empty_like, like)
        L.check(lib.ss_cache_attend(c.handle, self._ref, layer, N, n, C.byref(q), window, po, pl, ws.data_ptr(),
                                    need, _launch_stream(stream, dev), C.byref(o), lse.data_ptr()))
        if stream is not None:
            _used_on(stream, c.arena, self.tables, self.lengths, self.slots, queries, *(prior or ()))
            _returned_from(stream, out, lse)
        return out, lse
