"""A paged cache of keys and values in few bits: written as a model answers, read back, and attended
to.  Argument marshalling only, as in ``binding.py``; the entry points are ``bifeat_cache_*`` of
``include/bifeat.h``, which defines layout and arithmetic.  Ordinary calls go through the native module (``csrc/calls.cpp``) where
it is built; what it leaves goes through ctypes, behind the checks here."""
from __future__ import annotations

import ctypes as C
import functools
import math

from . import binding as _b
from .binding import EINVAL, _check, _dev_ptr, _dtype_code, _stream, _without_backward, _without_tangent, load_library


def _head_rows(t, heads: int, head_dim: int, name: str):
    """A [tokens, heads, head_dim] CUDA tensor as the library takes it: any token and head strides,
    columns next to each other."""
    if not t.is_cuda or t.dim() != 3 or t.shape[1] != heads or t.shape[2] != head_dim:
        raise ValueError(f"{name} must be a CUDA tensor [tokens, {heads}, {head_dim}]")
    s = t.stride()
    if s[2] != 1 and head_dim != 1:
        raise ValueError(f"{name}: a head's columns must be contiguous")
    return _b._CHeadRows(t.data_ptr(), s[0], s[1])


class PagedCache:
    """Owns a ``bifeat_cache`` handle: ``heads`` cached heads of ``head_dim`` columns in ``bits`` (4 or 8)
    bits, pages of ``page_size`` tokens.  The pages are the caller's: uint8 [pages, page_bytes].

    All calls take a batch: ``tables`` int32 [B, width], the pages of each sequence; ``lengths`` int64
    [B], its tokens, the call's own among them; ``indptr`` int64 [B + 1] or None, which rows of the
    call's arrays are whose (None: as many for every sequence).  The call is about the last of each
    sequence's tokens.  Work goes to the current stream; nothing is synchronised.  ``attend`` divides its work as if
    contexts were as long as ``tables`` is wide: pass ``tables[:, :most].contiguous()``, no wider than the
    longest context, where calls are short (a token over 300: 9.0 us, 16.3 by a table 4 times as wide).

    One object serves any streams and threads: ``attend`` has a workspace (68 MB) for each stream that it
    is called on, and one for captured calls (``reserve``).  CUDA graphs captured with one object must not be
    replayed at the same time, nor outlive it.  All tensors are of the current device."""

    def __init__(self, bits: int, heads: int, head_dim: int, page_size: int = 64):
        self._lib = load_library()
        h = C.c_void_p()
        _check(self._lib.bifeat_cache_create(C.byref(_b._CCacheSpec(bits, heads, head_dim, page_size)), C.byref(h)))
        self._h = h
        self.bits, self.heads, self.head_dim, self.page_size = int(bits), int(heads), int(head_dim), int(page_size)
        self.page_bytes = int(self._lib.bifeat_cache_page_bytes(h))
        self._scale = 1.0 / math.sqrt(self.head_dim)
        # what the native module's calls begin with: entry point, handle, sizes
        rest = (h.value, self.page_bytes, self.heads, self.head_dim)
        self._write, self._read, self._attend, self._append = (
            (_b._address(fn),) + rest
            for fn in (self._lib.bifeat_cache_write, self._lib.bifeat_cache_read, self._lib.bifeat_cache_attend, self._lib.bifeat_cache_append))

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        self._write = self._read = self._attend = self._append = (0,) * 5  # (no address of a destroyed object is left)
        if h:
            self._lib.bifeat_cache_destroy(h)

    def new_pages(self, count: int, device="cuda"):
        """Room for ``count`` pages.  What no token was written to is never looked at."""
        import torch
        return torch.empty((count, self.page_bytes), dtype=torch.uint8, device=device)

    def set_option(self, name: str, value: int) -> None:
        _check(self._lib.bifeat_cache_set_option(self._h, name.encode(), int(value)))

    def reserve(self) -> None:
        """The workspaces of ``attend`` on the current stream and of captured calls ahead of time (before a capture)."""
        _check(self._lib.bifeat_cache_reserve(self._h, _stream()))

    def _pages(self, pages, *others):
        import torch
        if not pages.is_cuda or pages.device.index != torch.cuda.current_device() or \
                any(t is not None and t.device != pages.device for t in others):
            raise ValueError("pages and the other tensors must be on the current CUDA device")
        if pages.dim() != 2 or pages.shape[1] != self.page_bytes:
            raise ValueError(f"pages must be [pages, {self.page_bytes}]")
        return _dev_ptr(pages, (torch.uint8,)), pages.shape[0]

    @staticmethod
    def _batch(tables, lengths, indptr, tokens):
        import torch
        if tables.dim() != 2 or lengths.shape != (tables.shape[0],):
            raise ValueError("tables must be [B, width], lengths [B]")
        B = tables.shape[0]
        if indptr is not None and indptr.shape != (B + 1,):
            raise ValueError("indptr must be [B + 1]")
        return _b._CCacheBatch(_dev_ptr(tables, (torch.int32,)), tables.shape[1], _dev_ptr(lengths, (torch.int64,)),
                               _dev_ptr(indptr, (torch.int64,)), B, tokens)

    def check(self, pages, tables, lengths, indptr=None, tokens=None) -> bool:
        """``bifeat_cache_check``: whether the batch is one that the calls may be given."""
        if tokens is None:
            tokens = int(indptr[-1]) if indptr is not None else tables.shape[0]
        rc = self._lib.bifeat_cache_check(self._h, self._pages(pages, tables, lengths, indptr)[1], C.byref(self._batch(tables, lengths, indptr, tokens)),
                                          _stream())
        if rc == EINVAL:
            return False
        _check(rc)
        return True

    def write(self, pages, k, v, tables, lengths, indptr=None) -> None:
        """Quantises k and v, [tokens, heads, head_dim], into the pages.  No gradient passes through codes."""
        if calls := _b._calls or _b._load_calls():
            r = calls.cache_write(*self._write, pages, k, v, tables, lengths, indptr)
            if r is not None:
                return _check(r)
        rows = [_head_rows(t, self.heads, self.head_dim, name) for t, name in ((k, "k"), (v, "v"))]
        if k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be alike")
        ptr, count = self._pages(pages, k, v, tables, lengths, indptr)
        _check(self._lib.bifeat_cache_write(self._h, ptr, count, C.byref(self._batch(tables, lengths, indptr, k.shape[0])),
                                            C.byref(rows[0]), C.byref(rows[1]), _dtype_code(k.dtype), _stream()))

    def append(self, pages, q, k, v, frequencies, tables, lengths, indptr=None, interleaved: bool = False, scale: float = 1.0):
        """``write`` of keys that are turned to their positions on the way; returns the queries, q [tokens, query heads, head_dim], turned
        with them (None for q None).  ``frequencies`` float32 [pairs], pairs <= head_dim / 2: radians a position of the column pairs
        (i, i + pairs), or (2 i, 2 i + 1) where ``interleaved``; columns from 2 * pairs on stay as they are.  ``scale``: of the turned
        columns.  Angles, and what becomes of keys and of 32-bit queries, are computed in 64 bits, queries of 16 bits in 32; a pair whose angle,
        position times frequency, is 2^50 or more in size becomes NaN.  No gradient passes through codes; where q or frequencies
        require one, going back through the output raises, and tensors with a tangent of forward-mode differentiation are refused."""
        if calls := _b._calls or _b._load_calls():
            r = calls.cache_append(*self._append, pages, q, k, v, frequencies, bool(interleaved), scale, tables, lengths, indptr)
            if r is not None:
                if r.__class__ is int:
                    _check(r)
                return None if r is True else r
        import torch
        _without_tangent("PagedCache.append has no forward-mode derivative", q, k, v, frequencies)
        if q is not None and (q.requires_grad or frequencies.requires_grad) and torch.is_grad_enabled():
            call = functools.partial(self.append, pages, q.detach(), k, v, frequencies.detach(), tables, lengths, indptr, interleaved, scale)
            return _without_backward().apply("PagedCache.append has no backward pass", call, q, frequencies)
        rows = [_head_rows(t, self.heads, self.head_dim, name) for t, name in ((k, "k"), (v, "v"))]
        if k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be alike")
        if frequencies.dim() != 1:
            raise ValueError("frequencies must be [pairs]")
        out, heads, q_rows = None, 0, _b._CHeadRows(None, 0, 0)
        if q is not None:
            if q.dim() != 3 or q.shape[0] != k.shape[0] or q.dtype != k.dtype:
                raise ValueError("q must be [tokens, query heads, head_dim] of k's tokens and type")
            heads = q.shape[1]
            q_rows = _head_rows(q, heads, self.head_dim, "q")
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        ptr, count = self._pages(pages, k, v, q, frequencies, tables, lengths, indptr)
        turn = _b._CTurn(_dev_ptr(frequencies, (torch.float32,)), frequencies.shape[0], bool(interleaved), scale)
        _check(self._lib.bifeat_cache_append(self._h, ptr, count, C.byref(self._batch(tables, lengths, indptr, k.shape[0])), C.byref(q_rows), heads,
                                             C.byref(rows[0]), C.byref(rows[1]), _dtype_code(k.dtype), C.byref(turn), _dev_ptr(out), _stream()))
        return out

    def read(self, pages, tables, lengths, tokens: int, indptr=None, dtype=None, out=None):
        """Keys and values of the last tokens of each sequence, ``tokens`` in all, as they stand in
        the cache: two [tokens, heads, head_dim] of ``dtype`` (float32)."""
        import torch
        if out is None and (calls := _b._calls or _b._load_calls()):
            r = calls.cache_read(*self._read, pages, tokens, _dtype_code(dtype or torch.float32), tables, lengths, indptr)
            if r is not None:
                if r.__class__ is int:
                    _check(r)
                return r
        shape = (tokens, self.heads, self.head_dim)
        if out is None:
            dtype = dtype or torch.float32
            out = (torch.empty(shape, dtype=dtype, device=pages.device), torch.empty(shape, dtype=dtype, device=pages.device))
        elif any(t.shape != shape for t in out) or out[0].dtype != out[1].dtype or dtype not in (None, out[0].dtype):
            raise ValueError("out must be two [tokens, heads, head_dim] of one dtype")
        ptr, count = self._pages(pages, *out, tables, lengths, indptr)
        _check(self._lib.bifeat_cache_read(self._h, ptr, count, C.byref(self._batch(tables, lengths, indptr, tokens)),
                                           _dev_ptr(out[0]), _dev_ptr(out[1]), _dtype_code(out[0].dtype), _stream()))
        return out

    def attend(self, pages, q, tables, lengths, indptr=None, scale=None, softcap: float = 0.0, window: int = 0, prefix=None,
               slopes=None, out=None):
        """Attention of the queries of each sequence's last tokens, q [tokens, query heads, head_dim], over
        what the cache holds of it, each up to itself.  ``scale`` of the products (1 / sqrt(head_dim));
        ``softcap`` c > 0: c * tanh(score / c); ``window`` w > 0: the last w positions only; ``prefix`` int64
        [B]: positions that all queries see; ``slopes`` float32 [query heads]: bias by distance.  Returns
        [tokens, query heads, head_dim] of q's dtype.  There is no backward pass: where q requires a gradient, going back
        through the output raises, and ``out`` is refused; a q with a tangent of forward-mode differentiation is refused."""
        scale = self._scale if scale is None else scale
        if out is None and (calls := _b._calls or _b._load_calls()):
            r = calls.cache_attend(*self._attend, pages, q, scale, softcap, window, prefix, slopes, tables, lengths, indptr)
            if r is not None:
                if r.__class__ is int:
                    _check(r)
                return r
        import torch
        _without_tangent("PagedCache.attend has no forward-mode derivative", q)
        if q.requires_grad and torch.is_grad_enabled():
            if out is not None:
                raise ValueError("attend has no backward pass: no out where q requires a gradient")
            args = (tables, lengths, indptr, scale, softcap, window, prefix, slopes)
            return _without_backward().apply("PagedCache.attend has no backward pass: the keys and values behind it are codes",
                                             lambda: self.attend(pages, q.detach(), *args), q)
        if q.dim() != 3:
            raise ValueError("q must be [tokens, query heads, head_dim]")
        heads = q.shape[1]
        rows = _head_rows(q, heads, self.head_dim, "q")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        elif out.shape != q.shape or out.dtype != q.dtype:
            raise ValueError("out must be like q")
        if prefix is not None and prefix.shape != (tables.shape[0],):
            raise ValueError("prefix must be [B]")
        if slopes is not None and slopes.shape != (heads,):
            raise ValueError("slopes must be [query heads]")
        ptr, count = self._pages(pages, q, out, tables, lengths, indptr, prefix, slopes)
        options = _b._CAttendOptions(scale, softcap, window,
                                     _dev_ptr(prefix, (torch.int64,)), _dev_ptr(slopes, (torch.float32,)))
        _check(self._lib.bifeat_cache_attend(self._h, ptr, count, C.byref(self._batch(tables, lengths, indptr, q.shape[0])),
                                             C.byref(rows), heads, _dtype_code(q.dtype), C.byref(options), _dev_ptr(out), _stream()))
        return out
