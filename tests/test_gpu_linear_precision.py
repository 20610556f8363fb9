"""How exact products with matrices in 4 bits are, by the root mean square of their errors: the same however many rows a call has, for rows
whose columns have a mean as for those that have none."""
import pytest

pytestmark = pytest.mark.gpu

MORE = {"f32": 0.0, "f16": 16.0, "bf16": 16.0}        # what the matrix cores' operands have of a code than the code
PIECES = {"f32": 3, "f16": 1, "bf16": 1}


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


def _rows(torch, g, kind, *shape):
    x = torch.randn(*shape, device="cuda", generator=g)
    return {"none": x, "one": x + 1, "positive": torch.relu(x)}[kind]


def _matrix(torch, layer, packed):
    """Codes, scale and minimum of each column [N, K] in 64 bits, from the documented layout."""
    N, K, group = layer.out_features, layer.in_features, layer.group
    rows, blocks = -(-N // 16), -(-K // 128)
    words = packed[:rows * blocks * 1024].view(torch.int32).view(rows, blocks, 4, 16, 4).long()      # [.][.][8 columns of a word][row][word]
    c = torch.arange(8, device="cuda")
    codes = words[..., None] >> 4 * (c // 2 + 4 * (c % 2)) & 15
    codes = codes.permute(0, 3, 1, 4, 2, 5).reshape(16 * rows, 128 * blocks)[:N, :K].double()
    levels = packed[rows * blocks * 1024:].view(torch.int32).view(rows, blocks * 128 // group, 16)
    levels = levels.transpose(1, 2).reshape(16 * rows, -1)[:N].repeat_interleave(group, 1)[:, :K].contiguous()
    scale, low = (levels << 16).view(torch.float32).double(), (levels & -65536).view(torch.float32).double()
    return codes, scale, low


def _rms(t):
    return float(t.double().square().mean().sqrt())


def _budget(torch, x, codes, scale, low, dtype):
    """The root mean square of what sums in 32 bits may be off by, with roundings that do not know of each other: 2^-23 of the number at hand each, which
    is more than three times what rounding to nearest is off by.  Of 128 columns (a group, or the groups that are added together): up to
    four adds a product of 16 columns and a piece of x, of numbers as large as the largest of the group's partial sums; then what the groups'
    minima and their scaled sums bring to the result, two adds a group of numbers as large as the result so far and what the minima bring together."""
    more, total, square = MORE[dtype], 0.0, 0.0
    for k in range(0, x.shape[1], 128):
        at = slice(k, k + 128)
        s, rest = scale[:, at], low[:, at] - more * scale[:, at]
        part = x[:, at, None] * (s * (codes[:, at] + more)).T[None] if x.shape[0] * s.numel() < 1 << 28 else None
        assert part is not None
        largest = part.cumsum(1).abs().amax(1)
        offset = x[:, at] @ rest.T
        groups = s.shape[1] // 32 + 1           # (at most: of 32 columns)
        square = square + 4 * PIECES[dtype] * 8 * largest.square() + 2 * groups * (torch.as_tensor(total, device="cuda").abs() + offset.abs()).square()
        total = total + x[:, at] @ (low[:, at] + s * codes[:, at]).T
    return 2.0 ** -23 * _rms(square.sqrt())


def _chain(K, group, want):
    return 2.0 ** -24 * (K / group + 1) ** 0.5 * _rms(want)


def _some(torch, T):
    """Rows whose errors are looked at: 64 of them, in all parts of a tile, the last among them."""
    return torch.linspace(0, T - 1, 64, device="cuda").round().long()


# Of 4096 rows by 1024 the tiles of 128 rows take less than the others, of 64 rows and fewer there are none.
CALLS = [(128, 4096, 4096, 1024), (32, 4096, 8192, 1024), (64, 4000, 5000, 1100)]


def _call(bf, torch, group, T, K, N, dtype, kind):
    g = torch.Generator(device="cuda").manual_seed(T + K)
    layer = bf.PackedLinear(N, K, group=group)
    packed = layer.pack(torch.randn(N, K, device="cuda", generator=g))
    x = _rows(torch, g, kind, T, K).to(_dtype(torch, dtype))
    some = _some(torch, T)
    few = x[some].contiguous()
    codes, scale, low = _matrix(torch, layer, packed)
    assert torch.equal((low + scale * codes).float(), layer.unpack(packed))
    want = few.double() @ (low + scale * codes).T
    return layer.multiply(packed, x)[some], layer.multiply(packed, few), want, few.double(), (codes, scale, low)


@pytest.mark.parametrize("kind", ["none", "one", "positive"])
@pytest.mark.parametrize("group,T,K,N", CALLS)
def test_many_32_bit_rows_are_as_exact_as_few(bf, torch, group, T, K, N, kind):
    """Both kernels bring minima and scaled sums of a group, or of the groups of 128 columns, to the result together.  Of four groups of 32 the
    minima bring 4 o at once and the sums take them back: roundings of sizes 4, 3, 2, 1 where groups one by one have four of size 1, 5.5 for 2; and the
    products are of 16 columns for 32, twice the adds, 1.4.  So less than 4 times the error, where results are one chain: of few rows the columns are
    split over waves, so that what rounds at the size of the result so far (two adds a group, of half the result's square on the average) is added."""
    many, few, want, *_ = _call(bf, torch, group, T, K, N, "f32", kind)
    a, b = _rms(many - want), _rms(few - want)
    assert a <= 4 * b + _chain(K, group, want), f"{a / _rms(want):.2e} of the result, of few rows {b / _rms(want):.2e}"


@pytest.mark.parametrize("group,T,K,N", CALLS)
def test_32_bit_rows_keep_32_bits_in_all_kernels(bf, torch, group, T, K, N):
    """Three bfloat16 are all of x: without the third the error would be more than the sums' roundings can explain."""
    many, few, want, x, matrix = _call(bf, torch, group, T, K, N, "f32", "none")
    x, want, many, few = x[::8], want[::8], many[::8], few[::8]
    allowed = _budget(torch, x, *matrix, "f32")
    codes, scale, low = matrix
    two = (x.float().view(torch.int32) & -256).view(torch.float32).double()
    assert _rms((two - x) @ (scale * codes).T) > 2 * allowed
    for got in (many, few):
        assert _rms(got - want) <= allowed, f"{_rms(got - want) / _rms(want):.2e} of the result, allowed {allowed / _rms(want):.2e}"


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["none", "one", "positive"])
@pytest.mark.parametrize("group,T,K,N", CALLS + [(32, 4096, 16384, 1024)])
def test_16_bit_results_are_off_by_their_rounding(bf, torch, group, T, K, N, kind, dtype):
    """Beside the result's rounding, which is what the exact result's own is off by, the sums' roundings count for little."""
    many, few, want, x, matrix = _call(bf, torch, group, T, K, N, dtype, kind)
    x, want, many, few = x[::8], want[::8], many[::8], few[::8]
    rounding, sums = _rms(want.to(many.dtype) - want), _budget(torch, x, *matrix, dtype)
    for got in (many, few):
        off = _rms(got - want)
        assert off <= (rounding ** 2 + sums ** 2) ** 0.5 * (1 + 2.0 ** -8), f"{off / rounding:.3f} of the rounding, the sums allowed {sums / rounding:.3f}"


# pairs by tiles of 16, and of 128
@pytest.mark.parametrize("joined", [False, True])
@pytest.mark.parametrize("kind", ["none", "one", "positive"])
@pytest.mark.parametrize("T", [12, 2000])
def test_experts_32_bit_rows(bf, torch, T, kind, joined):
    """An expert's rows are as exact as rows of one matrix (in tiles of 128 as above, of two groups of 64: sizes 2, 1 for two of size 1), and keep 32 bits."""
    E, k, K, N, group = 4, 2, 2048, 512, 64
    g = torch.Generator(device="cuda").manual_seed(T)
    layer, one = bf.PackedLinear(N, K, group=group, experts=E), bf.PackedLinear(N, K, group=group)
    packed = layer.pack(torch.randn(E, N, K, device="cuda", generator=g))
    x = _rows(torch, g, kind, T, K)
    ids = torch.randint(0, E, (T, k), device="cuda", dtype=torch.int32, generator=g)
    weights = torch.rand(T, k, device="cuda", generator=g)
    got = layer.multiply_experts(packed, x, ids, weights if joined else None)
    some = _some(torch, T)[::4]
    rows, ids, weights = x[some], ids[some].long(), weights[some]
    few, want, matrices = [], [], []
    for e in range(E):
        few.append(one.multiply(packed[e], rows))
        matrices.append(_matrix(torch, one, packed[e]))
        codes, scale, low = matrices[-1]
        want.append(rows.double() @ (low + scale * codes).T)
    at = torch.arange(len(some), device="cuda")[:, None]
    few, want = torch.stack(few, 1)[at, ids].double(), torch.stack(want, 1)[at, ids]
    # (a joined product is rounded once more in each multiply-add, which half a step of the largest covers)
    more = 0.0
    if joined:
        w = weights.double()[..., None]
        more = 2.0 ** -24 * 2 * _rms((w * want).abs().sum(1))
        few, want = (w * few).sum(1), (w * want).sum(1)
    off, of_few = _rms(got[some] - want), _rms(few - want)
    assert off <= 4 * of_few + _chain(K, group, want) + more, f"{off / _rms(want):.2e} of the result, of few rows {of_few / _rms(want):.2e}"
    if kind == "none" and not joined:
        allowed = max(_budget(torch, rows.double(), *m, "f32") for m in matrices)
        two = (rows.view(torch.int32) & -256).view(torch.float32).double()
        assert _rms((two - rows.double()) @ (matrices[0][0] * matrices[0][1]).T) > 2 * allowed
        assert off <= allowed, f"{off / _rms(want):.2e} of the result, allowed {allowed / _rms(want):.2e}"
