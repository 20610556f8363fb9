"""Matrices in 4 bits on the GPU against their definition in 64 bits: packed bit for bit, products of one row to many, experts' products."""
import numpy as np
import pytest

import linear_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16", "bf16"]
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}    # half the smallest step


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


def _weight(rng, *shape):
    return (rng.standard_normal(shape) * np.exp(0.5 * rng.standard_normal(shape[:-1] + (1,))) + 0.3 * rng.standard_normal(shape[:-1] + (1,))).astype(np.float32)


def _layer(bf, torch, rng, N, K, group):
    """A layer, its packed weights, and (values, size of a group's sums) in 64 bits."""
    q, s, m = ref.quantise(_weight(rng, N, K), group)
    layer = bf.PackedLinear(N, K, group=group)
    packed = torch.from_numpy(ref.pack(q, s, m, group)).cuda()
    at = np.arange(K) // group
    return layer, packed, ref.values(q, s, m, group), (31 * s.astype(np.float64) + np.abs(m))[:, at]


def _bound(K, x, size, want, dtype):
    """What sums in 32 bits may be off by: roundings along the longest chain of adds (32 columns of one matrix product, a group's and a row's
    products one after another, eight waves) of 2^-23 each, the matrix cores' adds being allowed a bit less than a rounding to nearest, of the sum
    of |x| times the largest that a code stands for in it; then the result's own rounding."""
    chain = 32 + 12 + 3 * (-(-K // 128)) + 8
    off = chain * 2.0 ** -23 * (np.abs(x) @ size.T)
    return off + (np.abs(want) + off) * HALF_ULP[dtype] + LEAST[dtype]


def _assert_close(got, want, bound, what=""):
    off = np.abs(got.astype(np.float64) - want)
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert (off <= bound).all(), f"{what} {(off > bound).sum()} of {off.size}, worst at {worst}: {got[worst]} for {want[worst]}, allowed {bound[worst]}"


# ------------------------------------------------------------------ pack and unpack

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 1), (16, 128), (17, 129), (100, 31), (5, 1001), (48, 640)])
def test_pack_matches_the_definition_bit_for_bit(bf, torch, dtype, group, N, K):
    rng = np.random.default_rng(N + K)
    w = torch.from_numpy(_weight(rng, N, K)).cuda().to(_dtype(torch, dtype))
    layer = bf.PackedLinear(N, K, group=group)
    q, s, m = ref.quantise(_host(w), group)
    want = ref.pack(q, s, m, group)
    out = torch.full((layer.bytes,), 0xa5, dtype=torch.uint8, device="cuda")
    assert layer.pack(w, out=out) is out
    got = out.cpu().numpy()
    assert got.size == want.size and np.array_equal(got, want), f"{(got != want).sum()} bytes differ"
    assert np.array_equal(layer.unpack(out).cpu().numpy(), ref.values(q, s, m, group).astype(np.float32))


def test_pack_of_special_groups(bf, torch):
    w = np.tile(np.linspace(-1, 2, 64, dtype=np.float32), (14, 1))
    w[1] = 0.25                                   # all alike, and bfloat16's
    w[2] = 0.1                                    # all alike
    w[3] = 0.0
    w[4] = -0.0
    w[5, 3] = np.nan
    w[6, 40] = np.inf
    w[7, 63] = -np.inf
    w[8] = np.linspace(-3e38, 3e38, 64)           # the range is no 32-bit number
    w[9] = -3.4e38                                # below bfloat16's least
    w[10] = np.linspace(0, 1e-39, 64)
    w[11] = 1e-30 * np.linspace(-1, 2, 64)
    w[12] = 1e37 * np.linspace(-1, 2, 64)
    w[13] = 1e-45
    layer = bf.PackedLinear(14, 64, group=64)
    q, s, m = ref.quantise(w, 64)
    p = layer.pack(torch.from_numpy(w).cuda())
    got = layer.unpack(p).cpu().numpy()
    assert np.isnan(got[5:10]).all() and np.isfinite(got[[0, 1, 2, 3, 4, 10, 11, 12, 13]]).all()
    assert (got[1] == 0.25).all() and not got[3:5].any()
    good = [0, 1, 2, 3, 4, 10, 11, 12, 13]
    assert np.array_equal(got[good], ref.values(q, s, m, 64)[good].astype(np.float32))
    for r in (0, 2, 11, 12):      # half a step (rounded up to 8 bits), and 32-bit roundings
        assert np.abs(got[r] - w[r]).max() <= s[r, 0] / 2 * (1 + 2.0 ** -20) + 2.0 ** -22 * np.abs(w[r]).max()
    # a spoilt row gives NaN, the others what they give without it; of row 12 the minimum times the sum of x is -6.4e38, which no 32-bit
    # sum holds, with a hundredth of x -6.4e36
    for size in (1.0, 0.01):
        x = torch.full((3, 64), size, device="cuda")
        y = layer.multiply(p, x).cpu().numpy()
        assert np.isnan(y[:, 5:10]).all() and np.isfinite(y[:, [r for r in good if r != 12 or size < 1]]).all()


def test_experts_are_packed_one_by_one(bf, torch):
    rng = np.random.default_rng(5)
    w = torch.from_numpy(_weight(rng, 3, 20, 200)).cuda()
    p = bf.PackedLinear(20, 200, group=64, experts=3).pack(w)
    one = bf.PackedLinear(20, 200, group=64)
    for e in range(3):
        assert torch.equal(p[e], one.pack(w[e]))
    # a transposed weight is taken as it is indexed
    assert torch.equal(one.pack(w[0].t().contiguous().t()), p[0])


# ------------------------------------------------------------------ products

SHAPES = [(1, 1, 1), (1, 128, 16), (1, 768, 768), (1, 1001, 37), (2, 4096, 33), (3, 31, 100), (15, 129, 17), (16, 256, 64), (17, 500, 48),
          (33, 96, 130), (40, 2048, 96), (64, 130, 256), (65, 640, 80), (100, 1000, 257), (129, 128, 128), (200, 300, 400), (257, 77, 129), (300, 2000, 300)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,K,N", SHAPES)
def test_multiply(bf, torch, dtype, group, T, K, N):
    rng = np.random.default_rng(T + K + N)
    layer, packed, value, size = _layer(bf, torch, rng, N, K, group)
    x = torch.from_numpy((rng.standard_normal((T, K)) + 0.5).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    # the result lies in the midst of other memory, which stays as it is
    room = torch.full((T + 2, N), 7.0, dtype=x.dtype, device="cuda")
    y = layer.multiply(packed, x, out=room[1:T + 1])
    h = _host(x).astype(np.float64)
    want = h @ value.T
    _assert_close(_host(y), want, _bound(K, h, size, want, dtype))
    assert (room[0] == 7).all() and (room[T + 1] == 7).all()
    assert torch.equal(layer.multiply(packed, x), y)                  # the same bits again


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 5, 30, 200])
def test_multiply_rows_that_lie_anywhere(bf, torch, dtype, T):
    rng = np.random.default_rng(T)
    K, N = 203, 50
    layer, packed, value, size = _layer(bf, torch, rng, N, K, 64)
    wide = torch.full((T * 407 + 9,), float("nan"), dtype=_dtype(torch, dtype), device="cuda")
    for stride, offset in ((407, 1), (204, 0), (203, 3), (208, 8)):
        x = torch.as_strided(wide, (T, K), (stride, 1), offset)
        wide.fill_(float("nan"))                                        # what lies between rows is not looked at
        x.copy_(torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)))
        h = _host(x).astype(np.float64)
        want = h @ value.T
        _assert_close(_host(layer.multiply(packed, x)), want, _bound(K, h, size, want, dtype), f"stride {stride}")
    # one row for all tokens, more dimensions, columns that are not next to each other, one row alone
    one = torch.from_numpy(rng.standard_normal(K).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    y = layer.multiply(packed, one.expand(T, K))
    assert torch.equal(y, y[:1].expand(T, N)) and torch.equal(layer.multiply(packed, one), layer.multiply(packed, one[None])[0])
    cube = torch.from_numpy(rng.standard_normal((T, 2, K)).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    assert torch.equal(layer.multiply(packed, cube), layer.multiply(packed, cube.reshape(-1, K)).view(T, 2, N))
    assert torch.equal(layer.multiply(packed, cube[:, 0].t().contiguous().t()), layer.multiply(packed, cube[:, 0].contiguous()))
    assert layer.multiply(packed, cube[:0]).shape == (0, 2, N)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [4, 20, 90, 200])
def test_rows_do_not_reach_each_other(bf, torch, dtype, T):
    rng = np.random.default_rng(T)
    K, N = 300, 70
    layer, packed, *_ = _layer(bf, torch, rng, N, K, 32)
    x = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    clean = layer.multiply(packed, x)
    bad = [0, T // 2, T - 1]
    for value in (float("nan"), float("inf"), -float("inf")):
        y = x.clone()
        y[bad, [0, 150, K - 1]] = value
        got = layer.multiply(packed, y)
        good = [t for t in range(T) if t not in bad]
        assert torch.equal(got[good], clean[good]) and not torch.isfinite(got[bad]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes_of_x_do_not_matter(bf, torch, dtype):
    rng = np.random.default_rng(8)
    layer, packed, value, size = _layer(bf, torch, rng, 64, 500, 128)
    for scale in (1e-30, 1e-6, 1e6, 1e30):
        for T in (3, 200):
            x = torch.from_numpy((scale * rng.standard_normal((T, 500))).astype(np.float32)).cuda().to(_dtype(torch, dtype))
            h = _host(x).astype(np.float64)
            want = h @ value.T
            _assert_close(_host(layer.multiply(packed, x)), want, _bound(500, h, size, want, dtype), str(scale))


@pytest.mark.parametrize("dtype,size", [("f16", 3e-6), ("f16", 3e-7), ("bf16", 1e-38), ("f32", 1e-37)])
@pytest.mark.parametrize("T", [3, 40, 2000])
def test_subnormal_rows(bf, torch, dtype, size, T):
    """Numbers below the type's smallest normal one are products' operands like others."""
    rng = np.random.default_rng(8)
    N = 2000 if T == 2000 else 64
    layer, packed, value, size_of = _layer(bf, torch, rng, N, 500, 128)
    x = torch.from_numpy((size * rng.standard_normal((T, 500))).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    h = _host(x).astype(np.float64)
    want = h @ value.T
    # fp32 sums have their own smallest steps too, 2^-150 to nearest, an addition; of a 32-bit number three bfloat16 are it but for what lies below
    # 2^-133, their smallest step, and so of a group's sum: twice that for each column, times the largest that a code stands for
    lost = 2.0 ** -132 * size_of.sum(1) if dtype == "f32" else 0.0
    _assert_close(_host(layer.multiply(packed, x)), want, _bound(500, h, size_of, want, dtype) + 700 * 2.0 ** -149 + lost)


# sizes at which tiles of many rows are taken, with the columns in one part and in four; few whole blocks of columns, and none
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group,T,K,N,stride", [(128, 1100, 1001, 3001, 1001), (64, 1300, 1152, 2500, 1160), (32, 1200, 1030, 3100, 1033), (128, 600, 8192, 2048, 8192),
                                                (32, 650, 8200, 2001, 8200), (64, 20000, 40, 3000, 47), (128, 20000, 9, 3003, 9), (128, 4096, 2304, 1000, 2304)])
def test_many_rows(bf, torch, dtype, group, T, K, N, stride):
    g = torch.Generator(device="cuda").manual_seed(T + K)
    layer = bf.PackedLinear(N, K, group=group)
    packed = layer.pack(torch.randn(N, K, device="cuda", generator=g) + 0.3 * torch.randn(N, 1, device="cuda", generator=g))
    wide = torch.full((T * stride + 3,), float("nan"), dtype=_dtype(torch, dtype), device="cuda")
    x = torch.as_strided(wide, (T, K), (stride, 1), 3)
    x.copy_(torch.randn(T, K, device="cuda", generator=g) + 0.5)
    room = torch.full((T + 2, N), 7.0, dtype=x.dtype, device="cuda")
    y = layer.multiply(packed, x, out=room[1:T + 1])
    value = layer.unpack(packed).double()
    want = x.double() @ value.T
    # as _bound; the largest that a code stands for in a group's sums: 31 scales and the minimum, 6 times the largest weight at most (a range of 15
    # scales has a weight of 7.5 of them at least: 31 scales are 4.2 of it, and the minimum is at most one)
    chain = 32 + 12 + 3 * (-(-K // 128)) + 8 + 16
    top = value.abs().view(N, K).nan_to_num()
    per = torch.stack([top[:, i:i + group].amax(1) for i in range(0, K, group)], 1).repeat_interleave(group, 1)[:, :K]
    off = chain * 2.0 ** -23 * (x.double().abs() @ (6 * per).T)
    assert ((y.double() - want).abs() <= off + (want.abs() + off) * HALF_ULP[dtype] + LEAST[dtype]).all()
    assert (room[0] == 7).all() and (room[T + 1] == 7).all() and torch.equal(layer.multiply(packed, x), y)
    # rows do not reach each other
    clean = y.clone()
    bad = [0, 130, T - 1]
    x[bad, [0, K // 2, K - 1]] = torch.tensor([float("nan"), float("inf"), -float("inf")], device="cuda").to(x.dtype)
    got = layer.multiply(packed, x)
    good = torch.ones(T, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.equal(got[good], clean[good]) and not torch.isfinite(got[bad]).any()


def test_32_bit_rows_keep_32_bits(bf, torch):
    """A weight of one code and x of full mantissas: the three pieces are all of x."""
    K, N = 64, 16
    layer = bf.PackedLinear(N, K, group=64)
    w = np.zeros((N, K), np.float32)
    w[np.arange(N), 3 * np.arange(N)] = 1.0             # code 15 of a scale of 1 / 15 rounded up: the weight is 15 scale
    packed = layer.pack(torch.from_numpy(w).cuda())
    scale = layer.unpack(packed)[0, 0].double()
    x = torch.randn(40, K, device="cuda")
    got = layer.multiply(packed, x).double()
    # columns of weight 0 add zeros; one product's rounding, one of the scale's
    want = x[:, 3 * torch.arange(N, device="cuda")].double() * scale
    assert ((got - want).abs() <= 2.0 ** -22 * want.abs() + 2.0 ** -23 * x.abs().sum(1, keepdim=True).double()).all()


def test_wide_and_long_matrices(bf, torch):
    for N, K, T in ((70000, 40, 3), (40, 70000, 3), (9, 70000, 100)):
        g = torch.Generator(device="cuda").manual_seed(N)
        layer = bf.PackedLinear(N, K, group=128)
        packed = layer.pack(torch.randn(N, K, device="cuda", generator=g))
        x = torch.randn(T, K, device="cuda", generator=g).half()
        value = layer.unpack(packed).double()
        want = x.double() @ value.T
        # the error of a sum of K terms, as it adds up at random (8 deviations), of terms up to 31 scale; the result's rounding
        off = 8 * 2.0 ** -23 * (x.double().square().sum(1, keepdim=True) * K).sqrt() * float(value.abs().max()) * 4
        assert ((layer.multiply(packed, x).double() - want).abs() <= off + want.abs() * 2.0 ** -11 + 2.0 ** -25).all()


# ------------------------------------------------------------------ experts

def _experts(bf, torch, rng, E, N, K, group):
    layer = bf.PackedLinear(N, K, group=group, experts=E)
    parts = [ref.quantise(_weight(rng, N, K), group) for _ in range(E)]
    packed = torch.from_numpy(np.stack([ref.pack(q, s, m, group) for q, s, m in parts])).cuda()
    at = np.arange(K) // group
    return layer, packed, [ref.values(q, s, m, group) for q, s, m in parts], [(31 * s.astype(np.float64) + np.abs(m))[:, at] for q, s, m in parts]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,K,N,group", [(1, 4, 1, 128, 32, 128), (1, 16, 8, 200, 65, 32), (7, 3, 2, 77, 40, 64), (33, 8, 3, 256, 48, 128), (64, 2, 2, 130, 100, 64),
                                             (100, 5, 4, 300, 64, 128), (200, 130, 6, 96, 33, 32), (500, 4, 2, 160, 130, 64), (90, 1, 1, 128, 16, 128),
                                             (3, 1024, 64, 40, 20, 32)])
@pytest.mark.parametrize("own_rows", [False, True])
@pytest.mark.parametrize("joined", [False, True])
def test_experts(bf, torch, dtype, T, E, k, K, N, group, own_rows, joined):
    rng = np.random.default_rng(T + E + K)
    layer, packed, values, sizes = _experts(bf, torch, rng, E, N, K, group)
    ids = rng.integers(0, E, (T, k))
    ids[rng.random((T, k)) < 0.1] = -1                      # none, or beyond the last
    ids[rng.random((T, k)) < 0.05] = E + 3
    if T > 2:
        ids[1] = -1
        ids[2] = ids[2, 0]                                  # one expert k times
    x = torch.from_numpy(rng.standard_normal((T, k, K) if own_rows else (T, K)).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    if own_rows:                                            # rows of choices that name none are not looked at
        x[torch.from_numpy((ids < 0) | (ids >= E)).cuda()] = float("nan")
    weights = rng.standard_normal((T, k)).astype(np.float32)
    shape = (T, N) if joined else (T, k, N)
    room = torch.full((T + 2,) + shape[1:], 7.0, dtype=x.dtype, device="cuda")
    args = (packed, x, torch.from_numpy(ids.astype(np.int32)).cuda(), torch.from_numpy(weights).cuda() if joined else None)
    got = layer.multiply_experts(*args, out=room[1:T + 1])
    h = _host(x).astype(np.float64)
    want, off = np.zeros((T, k, N)), np.zeros((T, k, N))
    for t in range(T):
        for j in range(k):
            e = ids[t, j]
            if 0 <= e < E:
                row = h[t, j] if own_rows else h[t]
                want[t, j] = values[e] @ row
                off[t, j] = (32 + 12 + 3 * (-(-K // 128)) + 8) * 2.0 ** -23 * (sizes[e] @ np.abs(row))
    if joined:
        # the products' errors and a rounding each, one an add
        off = (np.abs(weights)[..., None] * (off + (k + 2) * 2.0 ** -24 * np.abs(want))).sum(1)
        want = (weights.astype(np.float64)[..., None] * want).sum(1)
    _assert_close(_host(got), want, off + (np.abs(want) + off) * HALF_ULP[dtype] + LEAST[dtype])
    if T > 2:
        assert not got[1].any()
    assert (room[0] == 7).all() and (room[T + 1] == 7).all()
    assert torch.equal(layer.multiply_experts(*args), got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,E,k,K,N,group", [(450, 40, 4, 160, 1000, 64), (900, 16, 2, 300, 1030, 128), (600, 100, 3, 77, 900, 32), (7100, 3, 1, 96, 130, 32),
                                             (2000, 130, 8, 8, 65, 64), (700, 6, 3, 260, 1160, 32)])
@pytest.mark.parametrize("own_rows,joined", [(False, False), (True, True)])
def test_experts_of_many_pairs(bf, torch, dtype, T, E, k, K, N, group, own_rows, joined):
    test_experts(bf, torch, dtype, T, E, k, K, N, group, own_rows, joined)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("joined", [False, True])
def test_experts_tiles_of_every_fill(bf, torch, dtype, joined):
    """Experts with 1, 2, ... 140 pairs each."""
    rng = np.random.default_rng(5)
    E, K, N, group = 140, 136, 257, 64
    layer, packed, values, sizes = _experts(bf, torch, rng, E, N, K, group)
    ids = rng.permutation(np.repeat(np.arange(E), np.arange(1, E + 1)))[:, None]
    T = len(ids)
    assert T * 3 >= 14000 and T >= 16 * E
    x = torch.from_numpy(rng.standard_normal((T, K)).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    w = rng.random((T, 1)).astype(np.float32)
    h = _host(x).astype(np.float64)
    exact, size = np.zeros((T, N)), np.zeros((T, N))
    for e in range(E):
        at = ids[:, 0] == e
        exact[at] = h[at] @ values[e].T
        size[at] = _bound(K, np.abs(h[at]), sizes[e], exact[at], dtype)
    device_ids = torch.from_numpy(ids.astype(np.int32)).cuda()
    got = layer.multiply_experts(packed, x, device_ids, torch.from_numpy(w).cuda() if joined else None)
    if joined:      # (the product of the sum and the weight is rounded to 32 bits once more)
        exact, size = exact * w, size * w + np.abs(exact) * w * 2.0 ** -24 + LEAST[dtype]
    _assert_close(_host(got).reshape(T, N), exact, size)


@pytest.mark.parametrize("own_rows", [False, True])
def test_experts_rows_with_strides(bf, torch, own_rows):
    rng = np.random.default_rng(3)
    T, k, E, K, N = 21, 3, 4, 100, 40
    layer, packed, *_ = _experts(bf, torch, rng, E, N, K, 64)
    ids = torch.from_numpy(rng.integers(0, E, (T, k)).astype(np.int32)).cuda()
    wide = torch.full((T * 331 + 5,), float("nan"), dtype=torch.float16, device="cuda")
    view = torch.as_strided(wide, (T, k, K), (331, 105, 1), 3) if own_rows else torch.as_strided(wide, (T, K), (331, 1), 3)
    view.copy_(torch.randn(view.shape, device="cuda"))
    assert torch.equal(layer.multiply_experts(packed, view, ids), layer.multiply_experts(packed, view.contiguous(), ids))
    turned = view.transpose(-1, -2).contiguous().transpose(-1, -2)
    assert torch.equal(layer.multiply_experts(packed, turned, ids), layer.multiply_experts(packed, view.contiguous(), ids))
    assert layer.multiply_experts(packed, view[:0], ids[:0]).shape == (0, k, N)


def test_experts_all_tokens_to_one_and_to_none(bf, torch):
    rng = np.random.default_rng(4)
    E, K, N = 6, 256, 64
    layer, packed, *_ = _experts(bf, torch, rng, E, N, K, 128)
    one = bf.PackedLinear(N, K, group=128)
    for T in (5, 300, 3000):
        x = torch.randn(T, K, device="cuda").bfloat16()
        ids = torch.full((T, 2), 5, dtype=torch.int32, device="cuda")
        ids[:, 1] = 0
        y = layer.multiply_experts(packed, x, ids).double()
        for j, e in ((0, 5), (1, 0)):
            want = one.multiply(packed[e], x).double()
            assert ((y[:, j] - want).abs() <= 2.0 ** -7 * want.abs() + 1e-3).all()   # two kernels may round to neighbours
        assert not layer.multiply_experts(packed, x, torch.full_like(ids, -1)).any()
        assert not layer.multiply_experts(packed, x, torch.full_like(ids, 2 ** 31 - 1), torch.ones(T, 2, device="cuda")).any()


# ------------------------------------------------------------------ gradients, streams, graphs

@pytest.mark.parametrize("T", [1, 40, 300])
def test_outputs_beside_and_on_top_of_rows(bf, torch, T):
    rng = np.random.default_rng(T)
    N = K = 128
    layer, packed, values, size = _layer(bf, torch, rng, N, K, 64)
    rows = torch.randn(T, K, device="cuda").half()
    exact = _host(rows).astype(np.float64) @ values.T
    bound = _bound(K, np.abs(_host(rows).astype(np.float64)), size, exact, "f16")
    room = torch.zeros((2 * T + 1) * K, dtype=torch.float16, device="cuda")
    x = room[T * K:2 * T * K].view(T, K)
    x.copy_(rows)
    experts = bf.PackedLinear(N, K, group=64, experts=1)
    ids = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    for first in (T * K, 1, T * K + 127):
        out = room[first:first + T * K].view(T, N)
        with pytest.raises(bf.BifeatError):
            layer.multiply(packed, x, out=out)
        with pytest.raises(bf.BifeatError):
            experts.multiply_experts(packed[None], x, ids, out=out[:, None])
    beside = room[:T * K].view(T, N)
    _assert_close(_host(layer.multiply(packed, x, out=beside)), exact, bound)
    assert torch.equal(x, rows)
    _assert_close(_host(experts.multiply_experts(packed[None], x, ids, out=beside[:, None])[:, 0]), exact, bound)
    apart = torch.zeros(T, (T + 2) * K, dtype=torch.float16, device="cuda")     # out between the first row and the second
    apart[:, :K] = rows
    _assert_close(_host(layer.multiply(packed, apart[:, :K], out=apart[0, K:(T + 1) * K].view(T, N))), exact, bound)


def test_going_back_raises(bf, torch):
    rng = np.random.default_rng(0)
    layer, packed, *_ = _layer(bf, torch, rng, 16, 64, 64)
    x = torch.randn(3, 64, device="cuda", requires_grad=True)
    y = layer.multiply(packed, x)
    assert torch.equal(y, layer.multiply(packed, x.detach()))
    with pytest.raises(NotImplementedError):
        y.sum().backward()
    with pytest.raises(ValueError):
        layer.multiply(packed, x, out=torch.empty(3, 16, device="cuda"))
    with torch.no_grad():
        assert not layer.multiply(packed, x).requires_grad
    experts, packed, *_ = _experts(bf, torch, rng, 2, 16, 64, 64)
    ids, w = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, 1, device="cuda", requires_grad=True)
    for args in ((x, ids), (x.detach(), ids, w)):
        with pytest.raises(NotImplementedError):
            experts.multiply_experts(packed, *args).sum().backward()


def test_tensors_elsewhere_are_refused(bf, torch):
    layer = bf.PackedLinear(16, 64, group=64)
    packed = torch.zeros(layer.bytes, dtype=torch.uint8, device="cuda")
    x = torch.zeros(2, 64, device="cuda")
    for args in ((packed.cpu(), x), (packed, x.cpu()), (packed[:-1], x), (packed.view(torch.int8), x), (packed, x.double())):
        with pytest.raises(ValueError):
            layer.multiply(*args)
    with pytest.raises(bf.BifeatError):                 # 16-byte aligned
        layer.multiply(torch.zeros(layer.bytes + 1, dtype=torch.uint8, device="cuda")[1:], x)


def test_two_streams_at_once(bf, torch):
    rng = np.random.default_rng(1)
    layer, packed, *_ = _experts(bf, torch, rng, 8, 128, 512, 64)
    calls = []
    for i in range(2):
        x = torch.randn(400, 512, device="cuda").half()
        ids = torch.randint(0, 8, (400, 3), device="cuda", dtype=torch.int32)
        calls.append((x, ids, torch.rand(400, 3, device="cuda")))
    want = [layer.multiply_experts(packed, *c) for c in calls]
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (s, c) in enumerate(zip(streams, calls)):
            with torch.cuda.stream(s):
                got[i].append(layer.multiply_experts(packed, *c))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


@pytest.mark.parametrize("T", [1, 40, 300])
def test_captured_calls(bf, torch, T):
    rng = np.random.default_rng(2)
    layer, packed, *_ = _layer(bf, torch, rng, 96, 256, 64)
    experts, many, *_ = _experts(bf, torch, rng, 8, 64, 96, 32)
    x = torch.randn(T, 256, device="cuda").bfloat16()
    ids = torch.randint(0, 8, (T, 2), device="cuda", dtype=torch.int32)
    w = torch.rand(T, 2, device="cuda")

    def step():
        y = layer.multiply(packed, x)
        return y, experts.multiply_experts(many, y, ids), experts.multiply_experts(many, y, ids, w)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(torch.randn(T, 256, device="cuda"))
        ids.copy_(torch.randint(-1, 9, (T, 2), device="cuda"))
        want = step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


def test_the_example():
    """It runs, whole prompts and tokens one by one; of its numbers only that they are some."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_answers.py")
    spec = importlib.util.spec_from_file_location("packed_answers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    for bits in (4, 8):
        off = example.answer(bits, prompts=(70, 33, 5), tokens=6, chunk=32)
        assert len(off) == 3 and np.isfinite(off).all()
