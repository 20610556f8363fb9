"""Matrices in 4 bits, routing and turned rows without a GPU: sizes, the refusals that come before any GPU call, and the references that the
GPU tests compare with."""
import ctypes as C

import numpy as np
import pytest

import linear_reference as ref


@pytest.fixture(scope="module")
def bf():
    import os
    import paper_2207_14696_amd as m
    if not os.path.exists(m.library_path()):
        from paper_2207_14696_amd.build import build
        build()
    m.load_library()
    return m


def test_sizes_and_specs(bf):
    assert bf.PackedLinear(16, 128).bytes == 1024 + 64
    assert bf.PackedLinear(17, 129, group=32).bytes == 4 * (1024 + 4 * 64)
    assert bf.PackedLinear(1, 1, group=64, experts=5).bytes == 1024 + 128
    assert bf.PackedLinear(1 << 20, 1 << 20).bytes == (1 << 29) * 1088
    for bad in [(0, 1, 64), (1, 0, 64), (1, 1, 16), (1, 1, 256), (1, 1, 0), ((1 << 20) + 1, 1, 64), (1, (1 << 20) + 1, 64)]:
        with pytest.raises(bf.BifeatError) as e:
            bf.PackedLinear(*bad)
        assert e.value.status == bf.EINVAL
    for experts in (0, -1, 1025):
        with pytest.raises(bf.BifeatError):
            bf.PackedLinear(16, 16, 64, experts)


def test_sizes_that_32_bits_do_not_hold(bf):
    for sizes in ((1 << 32 | 16, 128), (16, 1 << 32 | 128), (16, 128, 1 << 32 | 64), (16, 128, 64, 1 << 32 | 2), (16 - (1 << 32), 128)):
        with pytest.raises(bf.BifeatError) as e:
            bf.PackedLinear(*sizes)
        assert e.value.status == bf.EINVAL


def test_linear_argument_errors_come_before_any_gpu_call(bf):
    from paper_2207_14696_amd.binding import _CExpertRows, _CLinearSpec
    lib = bf.load_library()

    def spec(n=32, k=64, group=64, experts=1):
        return C.byref(_CLinearSpec(n, k, group, experts))

    assert lib.bifeat_linear_bytes(None) == -1 and lib.bifeat_linear_bytes(spec(group=48)) == -1

    def pack(s=None, w=16, t=0, p=16):
        return lib.bifeat_linear_pack(s or spec(), w, t, p, None)

    assert pack(s=spec(n=0)) == pack(w=None) == pack(w=2) == pack(t=3) == pack(p=None) == pack(p=8) == -1
    assert lib.bifeat_linear_unpack(spec(), None, 16, None) == -1 and lib.bifeat_linear_unpack(spec(), 16, 2, None) == -1

    def multiply(s=None, p=16, x=16, stride=64, rows=3, t=0, out=16, room=16, size=1 << 40):
        return lib.bifeat_linear_multiply(s or spec(), p, x, stride, rows, t, out, room, size, None)

    def room(s=None, rows=3, t=0):
        return lib.bifeat_linear_workspace(s or spec(), rows, t)

    assert room(s=spec(experts=2)) == room(s=spec(group=1)) == room(rows=-1) == room(t=3) == -1 and room(rows=0) >= 0

    assert multiply(s=spec(experts=2)) == multiply(s=spec(k=-1)) == multiply(p=None) == multiply(p=8) == multiply(x=None) == multiply(x=2) == -1
    assert multiply(stride=-1) == multiply(rows=-1) == multiply(rows=1 << 31) == multiply(t=-1) == multiply(t=3) == -1
    assert multiply(out=None) == multiply(out=1, t=1) == multiply(x=1, t=2) == -1
    assert multiply(room=8) == -1
    assert multiply(rows=0, x=None, out=None, p=None, room=None, size=0) == 0

    def rows(x=16, ts=64, cs=0, ids=16, w=None, tokens=3, choices=2):
        return C.byref(_CExpertRows(x, ts, cs, ids, w, tokens, choices))

    def experts(s=None, p=16, r=None, t=0, out=16, room=16, size=1 << 20):
        return lib.bifeat_linear_experts(s or spec(experts=4), p, r or rows(), t, out, room, size, None)

    assert experts(s=spec(experts=0)) == experts(p=None) == experts(p=4) == experts(t=5) == experts(out=None) == experts(room=None) == -1
    assert experts(room=8) == experts(size=16) == experts(out=2) == -1
    for r in (rows(x=None), rows(x=2), rows(ts=-1), rows(cs=-1), rows(ids=None), rows(ids=2), rows(w=2), rows(tokens=-1), rows(choices=0),
              rows(choices=65), rows(tokens=1 << 30, choices=2)):
        assert experts(r=r) == -1
    assert experts(r=rows(tokens=0, x=None, ids=None), room=None, out=None, p=None) == 0
    assert lib.bifeat_linear_experts_workspace(None, rows()) == -1 and lib.bifeat_linear_experts_workspace(spec(), rows(choices=0)) == -1
    small, joined = (lib.bifeat_linear_experts_workspace(spec(experts=4), rows(w=w)) for w in (None, 16))
    assert joined == small + 6 * 32 * 4 and small % 16 == 0
    assert experts(r=rows(w=16), size=joined - 1) == -1


def test_outputs_on_top_of_rows_are_refused(bf):
    from paper_2207_14696_amd.binding import _CExpertRows, _CLinearSpec
    lib = bf.load_library()
    x, T, N, K = 1 << 30, 4000, 32, 64
    for dtype, e in ((0, 4), (1, 2), (2, 2)):
        row, outs = K * e, T * N * e

        def multiply(out, stride=K):
            return lib.bifeat_linear_multiply(C.byref(_CLinearSpec(N, K, 64, 1)), 16, x, stride, T, dtype, out, 16, 1 << 40, None)

        far = 10 ** 6
        assert multiply(x) == multiply(x - outs + e) == multiply(x + T * row - e) == multiply(x + row - e, far) == multiply(x + far * e - outs + e, far) == -1
        assert multiply(x + (T - 1) * far * e, far) == multiply(x, 0) == multiply(x + row - e, 0) == multiply(x, 1 << 62) == -1

        def experts(out, own=False, weights=None, token=2 * K, choice=K):
            r = _CExpertRows(x, token, choice if own else 0, 16, weights, T, 2)
            return lib.bifeat_linear_experts(C.byref(_CLinearSpec(N, K, 64, 4)), 16, C.byref(r), dtype, out, 16, 1 << 40, None)

        for w in (None, 16):
            assert experts(x, weights=w) == experts(x - e, weights=w) == experts(x + (2 * T - 1) * row - e, weights=w) == -1
            assert experts(x + 2 * T * row - e, True, w) == experts(x + far * e + row - e, True, w, 2 * far, far) == -1


def test_route_argument_errors_come_before_any_gpu_call(bf):
    from paper_2207_14696_amd.binding import _CRouteOptions
    lib = bf.load_library()

    def options(**kw):
        d = dict(experts=64, choices=4, sigmoid=0, groups=1, top_groups=1, group_two=0, renormalise=1, scale=1.0, bias=None)
        d.update(kw)
        return C.byref(_CRouteOptions(**d))

    def there(x=16, stride=64, t=0, tokens=3, o=None, ids=16, w=16):
        return lib.bifeat_route(x, stride, t, tokens, o or options(), ids, w, None)

    def back(x=16, stride=64, t=0, tokens=3, o=None, ids=16, w=16, out=16):
        return lib.bifeat_route_backward(x, stride, t, tokens, o or options(), ids, w, out, None)

    for call in (there, back):
        for o in (options(experts=0), options(experts=1025), options(choices=0), options(choices=65), options(experts=3, choices=4), options(groups=0),
                  options(groups=3), options(experts=130, groups=65), options(top_groups=0), options(groups=4, top_groups=5), options(sigmoid=2),
                  options(group_two=-1), options(renormalise=2), options(scale=float("nan")), options(scale=float("inf")), options(bias=2)):
            assert call(o=o) == -1
        assert call(x=None) == call(x=2) == call(stride=-1) == call(t=3) == call(tokens=-1) == call(ids=None) == call(ids=2) == -1
        assert call(w=None) == call(w=2) == call(tokens=1 << 31) == -1
        assert call(tokens=0, x=None, ids=None, w=None) == 0
    assert back(out=None) == back(out=2) == -1
    assert lib.bifeat_route(16, 64, 0, 3, None, 16, 16, None) == -1


def test_append_argument_errors_come_before_any_gpu_call(bf):
    from paper_2207_14696_amd.binding import _CCacheBatch, _CHeadRows, _CTurn
    lib = bf.load_library()
    c = bf.PagedCache(8, 2, 64, 16)

    def batch(**kw):
        d = dict(tables=16, table_width=4, lengths=16, indptr=None, sequences=2, tokens=2)
        d.update(kw)
        return C.byref(_CCacheBatch(**d))

    def rows(data=16, t=128, s=64):
        return C.byref(_CHeadRows(data, t, s))

    def turn(f=16, pairs=32, interleaved=0, scale=1.0):
        return C.byref(_CTurn(f, pairs, interleaved, scale))

    def append(h=c._h, pages=16, n=9, b=None, q=None, heads=4, k=None, v=None, t=0, f=None, out=16):
        return lib.bifeat_cache_append(h, pages, n, b or batch(), q or rows(), heads, k or rows(), v or rows(), t, f or turn(), out, None)

    assert append(h=None) == append(pages=8) == append(pages=None) == append(n=-1) == append(t=3) == append(heads=-1) == append(heads=65537) == -1
    for b in (batch(tokens=-1), batch(sequences=-1), batch(table_width=-1), batch(tokens=3), batch(lengths=None), batch(tables=None),
              batch(indptr=4), batch(tokens=1 << 31)):
        assert append(b=b) == -1
    for r in (rows(data=None), rows(data=2), rows(t=-1), rows(s=-1)):
        assert append(q=r) == append(k=r) == append(v=r) == -1
    for f in (turn(pairs=33), turn(pairs=-1), turn(f=None), turn(f=2), turn(interleaved=2), turn(scale=float("inf")), turn(scale=float("nan"))):
        assert append(f=f) == -1
    assert append(out=None) == append(out=2) == -1
    assert lib.bifeat_cache_append(c._h, 16, 9, batch(), rows(), 4, rows(), rows(), 0, None, 16, None) == -1
    assert append(b=batch(tokens=0, tables=None, lengths=None)) == 0


def test_python_refusals(bf):
    import torch
    x, host = torch.zeros(3, 64), torch.zeros(2, 1088, dtype=torch.uint8)
    a, e = bf.PackedLinear(16, 64), bf.PackedLinear(16, 64, experts=2)
    ids = torch.zeros(3, 2, dtype=torch.int32)
    for call in (lambda: a.multiply(host[0], x), lambda: a.multiply(host[0], torch.zeros(3, 65)), lambda: e.multiply(host, x),
                 lambda: a.multiply_experts(host[0], x, ids), lambda: e.multiply_experts(host, x, ids), lambda: e.multiply_experts(host, x, ids[:2]),
                 lambda: e.multiply_experts(host, torch.zeros(3, 3, 64), ids), lambda: e.multiply_experts(host, x, ids, torch.zeros(3, 3)),
                 lambda: a.multiply(host[0], x.double()), lambda: a.multiply(host[0], x.int()), lambda: a.pack(x), lambda: e.pack(torch.zeros(16, 64)),
                 lambda: a.unpack(host[0]), lambda: a.multiply(host[0], x, out=torch.zeros(3, 17)),
                 lambda: bf.route(x, 2), lambda: bf.route(x, 2, score="other"), lambda: bf.route(x, 2, group_score="most"),
                 lambda: bf.route(x, 2, bias=torch.zeros(63)), lambda: bf.route(torch.zeros(()), 1)):
        with pytest.raises(ValueError):
            call()


def test_reference_matrices():
    rng = np.random.default_rng(0)
    for group, N, K in ((32, 5, 70), (128, 18, 130), (64, 3, 1)):
        w = (rng.standard_normal((N, K)) * np.exp(rng.standard_normal((N, 1)))).astype(np.float32)
        q, s, m = ref.quantise(w, group)
        at = np.arange(K) // group
        assert (np.abs(ref.values(q, s, m, group) - w) <= 0.5001 * s[:, at] + 2.0 ** -22 * np.abs(w)).all()
        p = ref.pack(q, s, m, group)
        rows, blocks = -(-N // 16), -(-K // 128)
        assert p.size == rows * blocks * (1024 + 64 * 128 // group)
        for n, k in ((0, 0), (N - 1, K - 1), (N // 2, K // 3)):
            byte = ((n // 16) * blocks + k // 128) * 1024 + (n % 16 + 16 * (k % 32 // 8)) * 16 + k % 128 // 32 * 4
            word = int(p[byte:byte + 4].view(np.uint32)[0])
            assert word >> 4 * (k % 8 // 2 + 4 * (k % 2)) & 15 == q[n, k]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_reference_routing_gradient_against_differences(score, renormalise):
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((6, 12)), rng.standard_normal((6, 3))
    kw = dict(score=score, renormalise=renormalise, scale=1.7)
    ids, w = ref.route(x, 3, **kw)
    assert (np.diff(np.take_along_axis(x, ids, 1), axis=1) <= 0).all()
    want = ref.route_gradient(x, ids, g, **kw)
    step = 1e-6
    for e in range(12):
        # the choice held fixed: shares of the scores at `ids`
        def value(d):
            y = x.copy()
            y[:, e] += d
            p = np.take_along_axis(ref.scores_of(y, score), ids, 1)
            return (g * 1.7 * (p / p.sum(1, keepdims=True) if renormalise else p)).sum(1)
        # central differences: step^2 times third derivatives, and 2^-52 of the value over the step
        assert np.allclose((value(step) - value(-step)) / (2 * step), want[:, e], atol=2e-9)


def test_reference_turn_keeps_lengths_and_differences():
    rng = np.random.default_rng(2)
    x, f = rng.standard_normal((4, 2, 20)), 0.3 ** np.arange(8)
    for interleaved in (False, True):
        y = ref.turn(x, [0, 1, 7, 1000], f, interleaved)
        assert np.allclose(y[0], x[0]) and np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and np.array_equal(y[..., 16:], x[..., 16:])
        # products depend on the distance alone
        a, b = ref.turn(x[:2], [3, 9], f, interleaved), ref.turn(x[:2], [103, 109], f, interleaved)
        assert np.allclose((a[0] * a[1]).sum(-1), (b[0] * b[1]).sum(-1))


def test_the_product_kernels_spill_no_vector_registers(bf):
    import os
    from test_cache_abi import READELF, _kernels_of
    if not os.path.exists(READELF):
        pytest.skip("no llvm-readelf")
    kernels = [(n, s) for n, s in _kernels_of(bf.library_path()) if "linear_" in n or "route_" in n or "cache_append" in n]
    assert len(kernels) >= 100, len(kernels)
    assert not [k for k in kernels if k[1]]
