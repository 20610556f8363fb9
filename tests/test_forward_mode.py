"""Calls without a forward-mode derivative refuse tensors that carry a tangent; the output would have none, which is a derivative of zero."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad


@pytest.fixture(scope="module")
def bf():
    import os
    import paper_2207_14696_amd as m
    if not os.path.exists(m.library_path()):
        from paper_2207_14696_amd.build import build
        build()
    m.load_library()
    return m


def _calls(bf, device):
    """Calls by the tensor that may carry a tangent, and tensors for it."""
    r = lambda *shape: torch.randn(*shape, device=device)  # noqa: E731
    one, many = bf.PackedLinear(16, 32, group=32), bf.PackedLinear(16, 32, group=32, experts=2)
    packed = [torch.zeros(layer._lead() + (layer.bytes,), dtype=torch.uint8, device=device) for layer in (one, many)]
    ids, w, x, bias = torch.zeros(3, 2, dtype=torch.int32, device=device), r(3, 2), r(3, 32), r(32)
    c = bf.PagedCache(8, 2, 16, 16)
    pages = torch.zeros(1, c.page_bytes, dtype=torch.uint8, device=device)
    batch = (torch.zeros(1, 1, dtype=torch.int32, device=device), torch.tensor([3], device=device))
    q, k, v, f = r(3, 2, 16), r(3, 2, 16), r(3, 2, 16), r(8)
    return {
        "multiply": (lambda t: one.multiply(packed[0], t), x),
        "experts": (lambda t: many.multiply_experts(packed[1], t, ids), x),
        "joined experts": (lambda t: many.multiply_experts(packed[1], t, ids, w), x),
        "joined experts' weights": (lambda t: many.multiply_experts(packed[1], x, ids, t), w),
        "route": (lambda t: bf.route(t, 2), x),
        "route with a bias": (lambda t: bf.route(t, 2, score="sigmoid", bias=bias, groups=4, top_groups=2), x),
        "append q": (lambda t: c.append(pages, t, k, v, f, *batch), q),
        "append k": (lambda t: c.append(pages, q, t, v, f, *batch), k),
        "append v": (lambda t: c.append(pages, None, k, t, f, *batch), v),
        "append frequencies": (lambda t: c.append(pages, q, k, v, t, *batch), f),
        "attend": (lambda t: c.attend(pages, t, *batch), q),
    }


NAMES = ["multiply", "experts", "joined experts", "joined experts' weights", "route", "route with a bias", "append q", "append k", "append v",
         "append frequencies", "attend"]


def _refused(call, t):
    with forward_ad.dual_level():
        for requires in (False, True):
            x = forward_ad.make_dual(t.detach().requires_grad_(requires), torch.ones_like(t))
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call(x)
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                call(x)


@pytest.mark.parametrize("name", NAMES)
def test_tangents_are_refused_before_anything_else(bf, name):
    """No GPU: the refusal comes before that of tensors of the host."""
    _refused(*_calls(bf, "cpu")[name])


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_tangents_are_refused(bf, name):
    call, t = _calls(bf, "cuda")[name]
    want = call(t)
    _refused(call, t)
    same = lambda a, b: all(map(torch.equal, a, b)) if isinstance(a, tuple) else a is b is None or torch.equal(a, b)  # noqa: E731
    # without a tangent, or where they are switched off, the call is what it was
    with forward_ad.dual_level():
        assert same(call(t), want)
        with forward_ad._set_fwd_grad_enabled(False):
            assert same(call(forward_ad.make_dual(t, torch.ones_like(t))), want)
    if name in ("route", "route with a bias"):
        t = t.clone().requires_grad_(True)
        call(t)[1].sum().backward()
        assert t.grad is not None
