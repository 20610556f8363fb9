"""Routing on the GPU against its definition in 64 bits: choice, ties, masks, groups, weights, and the logits' gradient."""
import numpy as np
import pytest

import linear_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16", "bf16"]
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


@pytest.fixture(scope="module")
def bf():
    import paper_2207_14696_amd as m
    m.load_library()
    return m


@pytest.fixture(scope="module")
def torch():
    import torch as t
    return t


def _dtype(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def _host(t):
    return t.detach().float().cpu().numpy()


def _check(bf, torch, x, k, dtype, bias=None, grad=True, **kw):
    """One call, its choice, weights and gradient against the definition's."""
    device = torch.from_numpy(bias).cuda() if bias is not None else None
    x = x.detach().requires_grad_(grad)
    ids, weights = bf.route(x, k, bias=device, **kw)
    want_ids, want = ref.route(_host(x), k, bias=bias, **kw)
    got = ids.cpu().numpy()
    assert np.array_equal(got, want_ids), np.argwhere(got != want_ids)[:5]
    w = weights.detach().cpu().numpy()
    # scores of 64 bits, rounded to 32 once (an exponential and a sum of a thousand in 64 bits are off by less than 2^-40)
    off = np.abs(want) * (2.0 ** -24 + 2.0 ** -40) + 2.0 ** -150
    assert np.array_equal(np.isnan(w), np.isnan(want)) and (np.abs(w - want) <= off)[~np.isnan(want)].all()
    if not grad:
        return ids, weights
    g = np.random.default_rng(9).standard_normal(got.shape).astype(np.float32)
    dx, = torch.autograd.grad(weights, x, torch.from_numpy(g).cuda())
    assert dx.dtype == x.dtype and dx.shape == x.shape
    kw = {n: kw[n] for n in ("score", "renormalise", "scale") if n in kw}
    want = ref.route_gradient(_host(x), want_ids, g, **kw)
    spoilt = np.isnan(w).any(1)
    # terms cancel: of the size of the scale times |g|, off by 2^-40 of it
    off = np.abs(want) * (HALF_ULP[dtype] + 2.0 ** -23) + LEAST[dtype] + 2.0 ** -40 * kw.get("scale", 1.0) * np.abs(g).sum(1, keepdims=True)
    d = _host(dx)
    assert np.isnan(d[spoilt]).all() and (np.abs(d - want) <= off)[~spoilt].all()
    return ids, weights


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,T", [(1, 1, 3), (2, 1, 5), (8, 2, 33), (63, 5, 7), (64, 64, 9), (65, 8, 4), (100, 3, 30), (128, 8, 64), (256, 8, 50), (500, 10, 11),
                                   (512, 1, 6), (777, 33, 5), (1024, 64, 3)])
def test_choice_weights_and_gradient(bf, torch, dtype, score, E, k, T):
    rng = np.random.default_rng(E + k)
    x = torch.from_numpy((1.5 * rng.standard_normal((T, E))).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    for b in (None, bias):
        for renormalise in (True, False):
            _check(bf, torch, x, k, dtype, b, score=score, renormalise=renormalise, scale=2.5)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("group_score", ["best", "two"])
@pytest.mark.parametrize("E,groups,top,k", [(16, 4, 2, 3), (256, 8, 4, 8), (64, 64, 7, 5), (130, 2, 1, 20), (60, 12, 12, 4), (1024, 32, 3, 12), (36, 36, 1, 4), (96, 3, 2, 8),
                                            (384, 6, 3, 6)])
def test_groups(bf, torch, score, group_score, E, groups, top, k):
    rng = np.random.default_rng(E)
    x = torch.from_numpy(rng.standard_normal((40, E)).astype(np.float32)).cuda()
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32)
    for b in (None, bias):
        ids, _ = _check(bf, torch, x, k, "f32", b, score=score, groups=groups, top_groups=top, group_score=group_score)
        chosen = ids.cpu().numpy()
        per = E // groups
        assert all(len({e // per for e in row if e >= 0}) <= top for row in chosen)
        if k > top * per:
            assert (chosen[:, top * per:] == -1).all() and (chosen[:, :top * per] >= 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E", [10, 64, 200, 600])
def test_equal_logits_go_to_the_lowest_number(bf, torch, dtype, E):
    rng = np.random.default_rng(E)
    x = torch.from_numpy(rng.integers(-2, 3, (30, E)).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    x[0] = 0.5
    for score in ("softmax", "sigmoid"):
        ids, _ = _check(bf, torch, x, 6, dtype, score=score)
        assert ids[0].tolist() == list(range(6))
        _check(bf, torch, x, 6, dtype, np.zeros(E, np.float32), score=score)
        for group_score in ("best", "two"):
            _check(bf, torch, x, 6, dtype, score=score, groups=E // 2, top_groups=3, group_score=group_score) if E // 2 <= 64 else None
            _check(bf, torch, x, 6, dtype, score=score, groups=2, top_groups=1, group_score=group_score) if E >= 12 else None


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("groups", [1, 4])
def test_masked_experts(bf, torch, score, with_bias, groups):
    rng = np.random.default_rng(0)
    T, E, k = 12, 48, 5
    x = rng.standard_normal((T, E)).astype(np.float32)
    x[0] = -np.inf                              # none is to be had
    x[1, 1:] = -np.inf                          # one
    x[2, 3:] = -np.inf                          # fewer than asked for
    x[3, ::2] = -np.inf
    x[4] = np.finfo(np.float32).min             # the type's lowest is a logit like others
    x[5, 7:] = np.finfo(np.float32).min
    x[6, :24] = -np.inf                         # whole groups
    x[7, 0], x[7, 1:] = -np.inf, 80 * x[7, 1:]  # scores that vanish
    bias = (0.1 * rng.standard_normal(E)).astype(np.float32) if with_bias else None
    if with_bias:
        bias[5] = -np.inf                       # not to be had by any token
        bias[6] = np.nan
    for group_score in ("best", "two"):
        for renormalise in (True, False):
            ids, w = _check(bf, torch, torch.from_numpy(x).cuda(), k, "f32", bias, score=score, groups=groups, top_groups=min(groups, 2),
                            group_score=group_score, renormalise=renormalise)
            assert (ids[0] == -1).all() and not w[0].any() and (ids[1, 1:] == -1).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_spoilt_tokens(bf, torch, dtype):
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((9, 70)).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    clean = x.clone()
    x[2, 5] = float("nan")
    x[4, 69] = float("inf")
    x[6] = float("nan")
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            ids, w = _check(bf, torch, x, 3, dtype, score=score, renormalise=renormalise)
            good = [0, 1, 3, 5, 7, 8]
            want = bf.route(clean, 3, score=score, renormalise=renormalise)
            assert torch.equal(ids[good], want[0][good]) and torch.equal(w[good].detach(), want[1][good])
            assert int(ids[4, 0]) == 69 and (ids[6] == -1).all()


def test_chosen_scores_of_zero_have_no_gradient(bf, torch):
    """A bias, or groups by their two best, can choose experts whose softmax is 0 in 64 bits: weights of 0, which no logit moves."""
    x = torch.tensor([[0.0, -2000.0, -2001.0, -2000.0], [-2000.0, 0.0, -2000.0, -2000.5], [0.0, 1.0, 2.0, 1.5]], device="cuda")
    bias = np.array([0.0, 10.0, 10.0, 10.0], np.float32)
    _, w = _check(bf, torch, x, 2, "f32", bias)
    assert (w[0] == 0).all() and w[1, 0] == 1
    x = torch.tensor([[0.0, -np.inf, -np.inf, -np.inf, -800.0, -800.5, -801.0, -900.0]], device="cuda")
    bias = np.array([0, 0, 0, 0, 2, 2, 2, 2], np.float32)
    _, w = _check(bf, torch, x, 3, "f32", bias, groups=2, top_groups=1, group_score="two")
    assert (w == 0).all()


def test_scores_that_differ_in_their_last_digits(bf, torch):
    """Ranks of scores and biases that 32 bits would not tell apart."""
    E, T = 64, 50
    rng = np.random.default_rng(2)
    x = (0.5 + 2.0 ** -20 * rng.integers(0, 1000, (T, E))).astype(np.float32)
    bias = (1.0 + 2.0 ** -23 * rng.integers(0, 3, E)).astype(np.float32)
    for score in ("softmax", "sigmoid"):
        _check(bf, torch, torch.from_numpy(x).cuda(), 8, "f32", bias, score=score)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_lie_anywhere(bf, torch, dtype):
    wide = torch.full((20 * 150,), float("nan"), dtype=_dtype(torch, dtype), device="cuda")
    for E, stride, offset in ((100, 141, 3), (100, 101, 0), (128, 128, 1), (64, 72, 8)):
        wide.fill_(float("nan"))
        x = torch.as_strided(wide, (20, E), (stride, 1), offset)
        x.copy_(torch.randn(20, E, device="cuda"))
        _check(bf, torch, x, 4, dtype)
        _check(bf, torch, x.t().contiguous().t(), 4, dtype)
    cube = torch.randn(3, 5, 40, device="cuda").to(_dtype(torch, dtype))
    ids, w = bf.route(cube, 4)
    flat = bf.route(cube.view(15, 40), 4)
    assert torch.equal(ids.view(15, 4), flat[0]) and torch.equal(w.view(15, 4), flat[1]) and ids.dtype == torch.int32
    assert bf.route(cube[:0], 4)[0].shape == (0, 5, 4) and bf.route(cube[0, 0], 4)[0].shape == (4,)
    one = cube[0, 0].expand(7, 40)
    assert torch.equal(bf.route(one, 4)[0], bf.route(one.contiguous(), 4)[0])


def test_gradient_of_part_of_a_program(bf, torch):
    """Weights used twice, a weight's gradient that is not contiguous, a second derivative refused."""
    x = torch.randn(6, 32, device="cuda", requires_grad=True)
    ids, w = bf.route(x, 4, score="sigmoid")
    assert not ids.requires_grad
    g = torch.randn(4, 6, device="cuda").t()
    a, = torch.autograd.grad(w, x, g, retain_graph=True)
    b, = torch.autograd.grad((w * g).sum() + (w * 2 * g).sum(), x)
    assert torch.allclose(b, 3 * a, rtol=1e-5, atol=1e-7)       # sums of three 32-bit gradients
    _, w = bf.route(x, 4, score="sigmoid")
    d, = torch.autograd.grad(w.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()
    with torch.no_grad():
        assert not bf.route(x, 4)[1].requires_grad


def test_gradient_against_differences(bf, torch):
    rng = np.random.default_rng(4)
    x = rng.standard_normal((5, 20)).astype(np.float32)
    g = torch.from_numpy(rng.standard_normal((5, 3)).astype(np.float32)).cuda()
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            t = torch.from_numpy(x).cuda().requires_grad_(True)
            ids, w = bf.route(t, 3, score=score, renormalise=renormalise)
            dx, = torch.autograd.grad(w, t, g)
            step = 2.0 ** -7
            for e in range(20):
                values = []
                for sign in (1, -1):
                    y = x.copy()
                    y[:, e] += sign * step
                    i, v = bf.route(torch.from_numpy(y).cuda(), 3, score=score, renormalise=renormalise)
                    values.append(((v.double() * g.double()).sum(1), (i == ids).all(1)))
                same = values[0][1] & values[1][1]            # where the choice stays
                there = (values[0][0] - values[1][0]) / (2 * step)
                # step^2 / 6 times third derivatives (below 1 a weight), and weights' roundings over the step
                assert ((there - dx[:, e].double()).abs() <= step ** 2 / 6 * g.abs().sum(1) * 2 + g.abs().sum(1) * 2.0 ** -24 / step)[same].all()


def test_captured_routing_with_gradient(bf, torch):
    x = torch.randn(100, 256, device="cuda").requires_grad_(True)
    bias = 0.1 * torch.randn(256, device="cuda")
    g = torch.randn(100, 8, device="cuda")

    def step():
        ids, w = bf.route(x, 8, score="sigmoid", bias=bias, groups=8, top_groups=4, scale=2.5)
        return ids, w.detach(), torch.autograd.grad(w, x, g)[0]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        with torch.no_grad():
            x.copy_(torch.randn(100, 256, device="cuda"))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_refusals_on_the_device(bf, torch):
    x = torch.zeros(3, 16, device="cuda")
    for kw in (dict(choices=0), dict(choices=17), dict(choices=2, groups=3), dict(choices=2, groups=4, top_groups=5), dict(choices=2, scale=float("nan"))):
        with pytest.raises(bf.BifeatError):
            bf.route(x, **kw)
    for bad in (x.double(), x.int()):
        with pytest.raises(ValueError):
            bf.route(bad, 2)
    for bias in (torch.zeros(16), torch.zeros(16, device="cuda").half(), torch.zeros(32, device="cuda")[::2]):
        with pytest.raises(ValueError):
            bf.route(x, 2, bias=bias)


def test_numbers_that_32_bits_do_not_hold(bf, torch):
    x = torch.zeros(3, 16, device="cuda")
    for kw in (dict(choices=1 << 32 | 2), dict(choices=2, groups=1 << 32 | 4), dict(choices=2, groups=4, top_groups=(1 << 32) + 1), dict(choices=2 - (1 << 32))):
        with pytest.raises(bf.BifeatError):
            bf.route(x, **kw)
