"""Tokens routed to experts: ``bifeat_route`` of ``include/bifeat.h``, which defines scores, ranks, ties and weights, and
its gradient.  Argument marshalling only, as in ``binding.py``."""
from __future__ import annotations

import ctypes as C
import functools

from . import binding as _b
from .binding import EINVAL, _check, _dev_ptr, _dtype_code, _on_current_device, _stream, _without_tangent, load_library


_SCORES, _GROUP_SCORES = {"softmax": 0, "sigmoid": 1}, {"best": 0, "two": 1}


@functools.lru_cache(maxsize=None)
def _entries():
    lib = load_library()
    return _b._address(lib.bifeat_route), _b._address(lib.bifeat_route_backward)


def _rows(logits):
    rows = logits.reshape(-1, logits.shape[-1])
    return rows if rows.stride(1) == 1 or rows.shape[1] == 1 else rows.contiguous()


def _forward(logits, options):
    import torch
    rows, k = _rows(logits), options.choices
    ids = torch.empty(logits.shape[:-1] + (k,), dtype=torch.int32, device=logits.device)
    weights = torch.empty(ids.shape, dtype=torch.float32, device=logits.device)
    _on_current_device(logits)
    _check(load_library().bifeat_route(rows.data_ptr(), rows.stride(0), _dtype_code(logits.dtype), rows.shape[0], C.byref(options),
                                       ids.data_ptr(), weights.data_ptr(), _stream()))
    return ids, weights


@functools.lru_cache(maxsize=None)
def _function():
    import torch
    from torch.autograd.function import once_differentiable

    class Route(torch.autograd.Function):
        @staticmethod
        def forward(ctx, logits, options):
            ids, weights = _forward(logits, options)
            ctx.save_for_backward(logits, ids)
            ctx.options = options
            ctx.mark_non_differentiable(ids)
            return ids, weights

        @staticmethod
        @once_differentiable
        def backward(ctx, _, grad):
            logits, ids = ctx.saved_tensors
            rows, grad = _rows(logits), grad.contiguous()
            out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
            _on_current_device(logits, grad)
            _check(load_library().bifeat_route_backward(rows.data_ptr(), rows.stride(0), _dtype_code(logits.dtype), rows.shape[0],
                                                        C.byref(ctx.options), ids.data_ptr(), grad.data_ptr(), out.data_ptr(), _stream()))
            return out, None

    return Route


def route(logits, choices: int, score: str = "softmax", bias=None, groups: int = 1, top_groups: int = 1, group_score: str = "best",
          renormalise: bool = True, scale: float = 1.0):
    """Each token's ``choices`` experts and their weights from its logits [..., experts] (float32, float16 or bfloat16): ids
    int32 [..., choices], the first of the best rank, -1 where fewer are to be had; weights float32 [..., choices].

    ``score``: "softmax" or "sigmoid" of the logits.  ``bias`` float32 [experts] is added to the scores for the choice, not for the
    weights.  ``groups`` > 1: only the experts of the ``top_groups`` best groups of neighbours compete, a group being as good as
    its "best" expert or (``group_score`` "two") the sum of its two best.  ``renormalise``: weights are shares of their sum.  ``scale``: of the
    weights.  An expert whose logit is -infinity is not chosen.  Weights have a gradient in the logits (once); the choice and
    the bias have none.  Logits with a tangent of forward-mode differentiation are refused."""
    if score in _SCORES and group_score in _GROUP_SCORES and (calls := _b._calls or _b._load_calls()):
        r = calls.route(*_entries(), logits, choices, _SCORES[score], bias, groups, top_groups, _GROUP_SCORES[group_score], bool(renormalise), scale)
        if r is not None:
            if r.__class__ is int:
                _check(r)
            return r
    import torch
    if logits.dim() < 1 or score not in _SCORES or group_score not in _GROUP_SCORES:
        raise ValueError('logits must be [..., experts], score "softmax" or "sigmoid", group_score "best" or "two"')
    _without_tangent("route has no forward-mode derivative", logits)
    experts = logits.shape[-1]
    if bias is not None:
        if bias.shape != (experts,):
            raise ValueError("bias must be [experts]")
        _on_current_device(logits, bias)
    options = _b._CRouteOptions(experts, choices, _SCORES[score], groups, top_groups, _GROUP_SCORES[group_score], bool(renormalise), scale,
                                _dev_ptr(bias, (torch.float32,)))
    if (options.choices, options.groups, options.top_groups) != (choices, groups, top_groups):   # (numbers that 32 bits do not hold)
        _check(EINVAL)
    options.kept = bias     # (as long as a backward pass may need the options)
    if logits.requires_grad and torch.is_grad_enabled():
        return _function().apply(logits, options)
    return _forward(logits, options)
