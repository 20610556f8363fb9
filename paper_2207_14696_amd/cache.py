"""A paged cache of keys and values in few bits: written as a model answers, read back, and attended
to.  Argument marshalling only, as in ``binding.py``; the entry points are ``bifeat_cache_*`` of
``include/bifeat.h``, which defines layout and arithmetic.  Ordinary calls go through the native module (``csrc/calls.cpp``) where
it is built; what it leaves goes through ctypes, behind the checks here."""
from __future__ import annotations

import ctypes as C
import functools
import math

from . import binding as _b
from .binding import BF16, EINVAL, F16, F32, _check, _dev_ptr, _stream, load_library


def _type(dtype) -> int:
    import torch
    if dtype == torch.float16:
        return F16
    if dtype == torch.bfloat16:
        return BF16
    if dtype == torch.float32:
        return F32
    raise ValueError(f"unexpected dtype {dtype}: float32, float16 or bfloat16")


def _head_rows(t, heads: int, head_dim: int, name: str):
    """A [tokens, heads, head_dim] CUDA tensor as the library takes it: any token and head strides,
    columns next to each other."""
    if not t.is_cuda or t.dim() != 3 or t.shape[1] != heads or t.shape[2] != head_dim:
        raise ValueError(f"{name} must be a CUDA tensor [tokens, {heads}, {head_dim}]")
    s = t.stride()
    if s[2] != 1 and head_dim != 1:
        raise ValueError(f"{name}: a head's columns must be contiguous")
    return _b._CHeadRows(t.data_ptr(), s[0], s[1])


@functools.lru_cache(maxsize=None)
def _without_backward():
    """A function of autograd's graph around a call that has no backward pass: going back through it raises."""
    import torch

    class WithoutBackward(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, call):
            return call()

        @staticmethod
        def backward(ctx, grad):
            raise NotImplementedError("PagedCache.attend has no backward pass: the keys and values behind it are codes")

    return WithoutBackward


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
        self._write, self._read, self._attend = (
            (_b._address(fn),) + rest
            for fn in (self._lib.bifeat_cache_write, self._lib.bifeat_cache_read, self._lib.bifeat_cache_attend))

    def __del__(self):
        h, self._h = getattr(self, "_h", None), None
        self._write = self._read = self._attend = (0,) * 5  # (no address of a destroyed object is left)
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
                                            C.byref(rows[0]), C.byref(rows[1]), _type(k.dtype), _stream()))

    def read(self, pages, tables, lengths, tokens: int, indptr=None, dtype=None, out=None):
        """Keys and values of the last tokens of each sequence, ``tokens`` in all, as they stand in
        the cache: two [tokens, heads, head_dim] of ``dtype`` (float32)."""
        import torch
        if out is None and (calls := _b._calls or _b._load_calls()):
            r = calls.cache_read(*self._read, pages, tokens, _type(dtype or torch.float32), tables, lengths, indptr)
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
                                           _dev_ptr(out[0]), _dev_ptr(out[1]), _type(out[0].dtype), _stream()))
        return out

    def attend(self, pages, q, tables, lengths, indptr=None, scale=None, softcap: float = 0.0, window: int = 0, prefix=None,
               slopes=None, out=None):
        """Attention of the queries of each sequence's last tokens, q [tokens, query heads, head_dim], over
        what the cache holds of it, each up to itself.  ``scale`` of the products (1 / sqrt(head_dim));
        ``softcap`` c > 0: c * tanh(score / c); ``window`` w > 0: the last w positions only; ``prefix`` int64
        [B]: positions that all queries see; ``slopes`` float32 [query heads]: bias by distance.  Returns
        [tokens, query heads, head_dim] of q's dtype.  There is no backward pass: where q requires a gradient, going back
        through the output raises, and ``out`` is refused."""
        scale = self._scale if scale is None else scale
        if out is None and (calls := _b._calls or _b._load_calls()):
            r = calls.cache_attend(*self._attend, pages, q, scale, softcap, window, prefix, slopes, tables, lengths, indptr)
            if r is not None:
                if r.__class__ is int:
                    _check(r)
                return r
        import torch
        if q.requires_grad and torch.is_grad_enabled():
            if out is not None:
                raise ValueError("attend has no backward pass: no out where q requires a gradient")
            args = (tables, lengths, indptr, scale, softcap, window, prefix, slopes)
            return _without_backward().apply(q, lambda: self.attend(pages, q.detach(), *args))
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
                                             C.byref(rows), heads, _type(q.dtype), C.byref(options), _dev_ptr(out), _stream()))
        return out
