"""Products with matrices in 4 bits, for a model's layers and for its experts.  Argument marshalling only, as in ``binding.py``;
the entry points are ``bifeat_linear_*`` of ``include/bifeat.h``, which defines layout and arithmetic.  Ordinary calls go
through the native module (``csrc/calls.cpp``) where it is built."""
from __future__ import annotations

import ctypes as C

from . import binding as _b
from .binding import EINVAL, _check, _dev_ptr, _dtype_code, _on_current_device, _stream, _without_backward, _without_tangent, load_library

_WHY = "PackedLinear has no backward pass: its weights are codes"
_FORWARD = "PackedLinear has no forward-mode derivative"


class PackedLinear:
    """A layer of ``out_features`` x ``in_features`` weights in 4 bits, with a scale and a minimum for each ``group`` (32, 64 or
    128) columns of a row; or, with ``experts``, that many of one size.  The packed weights are the caller's: uint8 [bytes], or
    [experts, bytes].  Nothing is kept between calls, so any streams, threads and graphs may share one object.  Work goes to the
    current stream; nothing is synchronised.  All tensors are of the current device."""

    def __init__(self, out_features: int, in_features: int, group: int = 128, experts: int | None = None):
        self._lib = load_library()
        self._spec = _b._CLinearSpec(out_features, in_features, group, 1 if experts is None else experts)
        self.bytes = int(self._lib.bifeat_linear_bytes(C.byref(self._spec)))
        if self.bytes < 0 or (self._spec.out_features, self._spec.in_features, self._spec.group) != (out_features, in_features, group) or \
                self._spec.experts != (1 if experts is None else experts):  # (sizes that 32 bits do not hold)
            _check(EINVAL)
        self.out_features, self.in_features, self.group = int(out_features), int(in_features), int(group)
        self.experts = None if experts is None else int(experts)
        # what the native module's calls begin with: entry points, sizes
        sizes = (self.out_features, self.in_features, self.group)
        self._multiply = (_b._address(self._lib.bifeat_linear_workspace), _b._address(self._lib.bifeat_linear_multiply), *sizes, self.bytes)
        self._by_experts = (_b._address(self._lib.bifeat_linear_experts_workspace), _b._address(self._lib.bifeat_linear_experts), *sizes,
                            self.experts, self.bytes)

    def _lead(self):
        return () if self.experts is None else (self.experts,)

    def _packed(self, packed, *others):
        import torch
        _on_current_device(packed, *others)
        if tuple(packed.shape) != self._lead() + (self.bytes,):
            raise ValueError(f"packed must be uint8 {list(self._lead() + (self.bytes,))}")
        return _dev_ptr(packed, (torch.uint8,))

    def pack(self, weight, out=None):
        """Quantises weight, [out_features, in_features] (with experts: [experts, ...]) of float32, float16 or bfloat16."""
        import torch
        if tuple(weight.shape) != self._lead() + (self.out_features, self.in_features):
            raise ValueError(f"weight must be {list(self._lead() + (self.out_features, self.in_features))}")
        weight = weight.detach().contiguous()
        if out is None:
            out = torch.empty(self._lead() + (self.bytes,), dtype=torch.uint8, device=weight.device)
        ptr = self._packed(out, weight)
        _check(self._lib.bifeat_linear_pack(C.byref(self._spec), _dev_ptr(weight), _dtype_code(weight.dtype), ptr, _stream()))
        return out

    def unpack(self, packed):
        """The weights that the codes stand for, float32."""
        import torch
        out = torch.empty(self._lead() + (self.out_features, self.in_features), dtype=torch.float32, device=packed.device)
        _check(self._lib.bifeat_linear_unpack(C.byref(self._spec), self._packed(packed), _dev_ptr(out), _stream()))
        return out

    def multiply(self, packed, x, out=None):
        """x [..., in_features] times the matrix's rows: [..., out_features] of x's type (float32, float16 or bfloat16).  Rows may lie any
        distance apart, their columns next to each other.  There is no backward pass: where x requires a gradient, going back
        through the output raises, and ``out`` is refused; an x with a tangent of forward-mode differentiation is refused.  ``out`` shares no memory with x (refused too)."""
        if out is None and self.experts is None and (calls := _b._calls or _b._load_calls()):
            r = calls.linear_multiply(*self._multiply, packed, x)
            if r is not None:
                if r.__class__ is int:
                    _check(r)
                return r
        import torch
        if self.experts is not None:
            raise ValueError("a layer of experts: multiply_experts")
        if x.dim() < 1 or x.shape[-1] != self.in_features:
            raise ValueError(f"x must be [..., {self.in_features}]")
        _without_tangent(_FORWARD, x)
        if x.requires_grad and torch.is_grad_enabled():
            if out is not None:
                raise ValueError(_WHY + ": no out where x requires a gradient")
            return _without_backward().apply(_WHY, lambda: self.multiply(packed, x.detach()), x)
        code = _dtype_code(x.dtype)
        rows = x.reshape(-1, self.in_features)
        if rows.stride(1) != 1 and self.in_features != 1:
            rows = rows.contiguous()
        shape = x.shape[:-1] + (self.out_features,)
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=x.device)
        elif out.shape != shape or out.dtype != x.dtype:
            raise ValueError(f"out must be {list(shape)} of x's type")
        ptr = self._packed(packed, rows, out)
        need = self._lib.bifeat_linear_workspace(C.byref(self._spec), rows.shape[0], code)
        if need < 0:
            _check(int(need))
        room = torch.empty(need, dtype=torch.uint8, device=x.device)
        _check(self._lib.bifeat_linear_multiply(C.byref(self._spec), ptr, rows.data_ptr(), rows.stride(0), rows.shape[0], code, _dev_ptr(out),
                                                room.data_ptr(), need, _stream()))
        return out

    def multiply_experts(self, packed, x, ids, weights=None, out=None):
        """Each token by the matrices of its experts: x [tokens, in_features], or [tokens, choices, in_features] where each choice has a row of its
        own; ids int32 [tokens, choices], as ``route`` gives them (an id outside [0, experts) names none and gives zeros).  Returns
        [tokens, choices, out_features] of x's type, or with ``weights`` float32 [tokens, choices] their weighted sum,
        [tokens, out_features].  Takes memory for the time of the call (``bifeat_linear_experts_workspace`` has the number): 4 bytes a place of a
        pair of a token and a choice, each expert's places filled up to a multiple of 16, or of 128 where pairs are many; there 8 bytes a group of
        each row of x besides; with weights 4 * out_features a pair.  No backward pass, and an ``out`` of its own memory, as ``multiply``."""
        if out is None and self.experts is not None and (calls := _b._calls or _b._load_calls()):
            r = calls.linear_experts(*self._by_experts, packed, x, ids, weights)
            if r is not None:
                if r.__class__ is int:
                    _check(r)
                return r
        import torch
        if self.experts is None:
            raise ValueError("a layer of one matrix: multiply")
        if ids.dim() != 2 or x.dim() not in (2, 3) or x.shape[0] != ids.shape[0] or x.shape[-1] != self.in_features or \
                (x.dim() == 3 and x.shape[1] != ids.shape[1]):
            raise ValueError(f"ids must be [tokens, choices], x [tokens, {self.in_features}] or [tokens, choices, {self.in_features}]")
        if weights is not None and weights.shape != ids.shape:
            raise ValueError("weights must be like ids")
        _without_tangent(_FORWARD, x, weights)
        if torch.is_grad_enabled() and (x.requires_grad or (weights is not None and weights.requires_grad)):
            if out is not None:
                raise ValueError(_WHY + ": no out where x or weights require a gradient")
            return _without_backward().apply(
                _WHY, lambda: self.multiply_experts(packed, x.detach(), ids, None if weights is None else weights.detach()), x, weights)
        code = _dtype_code(x.dtype)
        if x.stride(-1) != 1 and self.in_features != 1:
            x = x.contiguous()
        tokens, choices = ids.shape
        shape = (tokens, self.out_features) if weights is not None else (tokens, choices, self.out_features)
        if out is None:
            out = torch.empty(shape, dtype=x.dtype, device=x.device)
        elif out.shape != shape or out.dtype != x.dtype:
            raise ValueError(f"out must be {list(shape)} of x's type")
        ptr = self._packed(packed, x, ids, weights, out)
        rows = _b._CExpertRows(x.data_ptr(), x.stride(0), x.stride(1) if x.dim() == 3 else 0, _dev_ptr(ids, (torch.int32,)),
                               _dev_ptr(weights, (torch.float32,)), tokens, choices)
        need = self._lib.bifeat_linear_experts_workspace(C.byref(self._spec), C.byref(rows))
        if need < 0:
            _check(int(need))
        room = torch.empty(need, dtype=torch.uint8, device=x.device)
        _check(self._lib.bifeat_linear_experts(C.byref(self._spec), ptr, C.byref(rows), code, _dev_ptr(out), room.data_ptr(), need, _stream()))
        return out
