"""Keys turned to their positions on their way into the paged cache, and queries beside them, against the definition in 64 bits."""
import numpy as np
import pytest

import cache_reference as ref
from linear_reference import turn
from test_gpu_cache import HALF_ULP, TYPES, Batch, _dtype, _host, _random_bytes, _rows, bf, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


def _frequencies(torch, pairs):
    return (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).float().cuda()


def _positions(batch):
    """Position of every token, negative before its sequence's beginning."""
    return np.concatenate([np.arange(m - n, m) for m, n in zip(batch.lengths, batch.news)] or [np.zeros(0)]).astype(np.int64)


def _check(bf, torch, batch, bits, heads, group, d, ps, dtype, layout, pairs, interleaved, scale=1.0, seed=0, frequencies=None):
    rng = np.random.default_rng(seed)
    c = bf.PagedCache(bits, heads, d, ps)
    want = _random_bytes(rng, batch.count, c.page_bytes)
    pages = torch.from_numpy(want.copy()).cuda()
    q = _rows(torch, rng, batch.T, heads * group, d, dtype, layout)
    k, v = (_rows(torch, rng, batch.T, heads, d, dtype, layout) for _ in range(2))
    f = _frequencies(torch, pairs) if frequencies is None else frequencies
    got_q = c.append(pages, q, k, v, f, batch.d_tables, batch.d_lengths, batch.d_indptr, interleaved=interleaved, scale=scale)
    at, hf = _positions(batch), f.cpu().numpy()
    hk, hv = turn(_host(k), at, hf, interleaved, scale).astype(np.float32), _host(v)
    oracle = ref.Pages(want, bits, heads, d, ps)
    for t, page, slot in batch.places():
        for h in range(heads):
            oracle.put(page, slot, h, 0, hk[t, h])
            oracle.put(page, slot, h, 1, hv[t, h])
    got = pages.cpu().numpy()
    assert np.array_equal(got, want), f"{(got != want).sum()} bytes differ"
    want_q = turn(_host(q), at, hf, interleaved, scale)
    want_q[at < 0] = 0.0
    assert got_q.dtype == q.dtype and got_q.shape == q.shape and got_q.is_contiguous()
    # rounded to 32 bits, then to the type; queries of 16 bits in numbers of 32: cosine and sine rounded (2^-25 of them: they are below 1, times the
    # scale), products (2^-24) and their sum (2^-24), so within 2^-22 of scale (|u| + |w|),
    # which is at most twice the row's largest
    off = np.abs(_host(got_q) - want_q)
    turned = 0.0 if dtype == "f32" else 2.0 ** -22 * scale * np.abs(_host(q)).max(-1, keepdims=True) * 2
    assert (off <= (np.abs(want_q) + turned) * (HALF_ULP[dtype] + 2.0 ** -24 + 2.0 ** -40) + turned + 2.0 ** -25 * (dtype == "f16") + 1e-13).all()
    return c, pages


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype,heads,group,d,ps,layout,pairs", [
    ("f16", 12, 1, 64, 16, "joint", 32), ("bf16", 8, 4, 128, 64, "packed", 64), ("f32", 2, 3, 100, 16, "odd", 50), ("f16", 1, 8, 256, 32, "heads_first", 128),
    ("bf16", 3, 1, 37, 16, "odd", 18), ("f32", 5, 2, 1, 16, "packed", 0), ("f16", 7, 1, 129, 128, "odd", 16), ("bf16", 2, 2, 8, 1024, "heads_first", 3),
    ("bf16", 4, 1, 128, 16, "joint", 16), ("f32", 1, 1, 2, 16, "odd", 1), ("f16", 2, 5, 80, 32, "joint", 0), ("f32", 3, 1, 200, 16, "packed", 41)])
def test_append_matches_the_definition_bit_for_bit(bf, torch, bits, interleaved, dtype, heads, group, d, ps, layout, pairs):  # noqa: F811
    batch = Batch(torch, [1, ps, 2 * ps + 5, 40, 3, ps + 1, 0], [1, 3, ps + 7, 0, 5, 1, 2], ps)
    _check(bf, torch, batch, bits, heads, group, d, ps, dtype, layout, pairs, interleaved, scale=1.0 if d % 2 else 1.25, seed=d + bits)


def test_far_positions(bf, torch):  # noqa: F811
    """Angles of a million radians: a table in pages that few sequences' ends lie in."""
    ps, far = 1024, 1 << 20
    lengths = [far, far - 7, far // 2 + 9]
    assert all((m - 1) // ps == (m - 4) // ps for m in lengths)      # (a sequence's new tokens in one page, the only one that its table names)
    batch = Batch(torch, [4, 4, 4], [4, 4, 4], ps)
    width = far // ps
    tables = torch.full((3, width), -7, dtype=torch.int32, device="cuda")
    for b, m in enumerate(lengths):
        tables[b, (m - 1) // ps] = b
    batch.d_tables, batch.d_lengths, batch.lengths = tables, torch.tensor(lengths, device="cuda"), lengths
    batch.places = lambda: ((4 * b + i, b, (m - 4 + i) % ps) for b, m in enumerate(lengths) for i in range(4))
    for interleaved in (False, True):
        _check(bf, torch, batch, 8, 2, 2, 64, ps, "f32", "joint", 32, interleaved)
        _check(bf, torch, batch, 8, 2, 2, 64, ps, "bf16", "joint", 32, interleaved, frequencies=torch.linspace(0, 3, 32, device="cuda"))


@pytest.mark.parametrize("tokens", [1, 2, 300, 5000])
def test_append_of_any_number_of_tokens(bf, torch, tokens):  # noqa: F811
    batch = Batch(torch, [tokens + 11], [tokens], 16)
    _check(bf, torch, batch, 8, 1, 1, 32, 16, "bf16", "joint", 16, False)


def test_untouched_columns_and_written_as_write_does(bf, torch):  # noqa: F811
    """No pairs: what ``write`` writes, and the queries as they were; no queries: None."""
    batch = Batch(torch, [20, 5], [7, 5], 16)
    c = bf.PagedCache(4, 2, 48, 16)
    rng = np.random.default_rng(0)
    q, k, v = _rows(torch, rng, 12, 4, 48, "bf16"), _rows(torch, rng, 12, 2, 48, "bf16"), _rows(torch, rng, 12, 2, 48, "bf16")
    a = torch.zeros(batch.count, c.page_bytes, dtype=torch.uint8, device="cuda")
    b = a.clone()
    none = torch.zeros(0, device="cuda")
    got = c.append(a, q, k, v, none, batch.d_tables, batch.d_lengths, batch.d_indptr)
    c.write(b, k, v, batch.d_tables, batch.d_lengths, batch.d_indptr)
    assert torch.equal(got, q) and torch.equal(a, b)
    a.zero_()
    assert c.append(a, None, k, v, none, batch.d_tables, batch.d_lengths, batch.d_indptr) is None and torch.equal(a, b)
    f = _frequencies(torch, 24)
    full = c.append(a, q, k, v, f, batch.d_tables, batch.d_lengths, batch.d_indptr)
    c.append(b, None, k, v, f, batch.d_tables, batch.d_lengths, batch.d_indptr)
    assert torch.equal(a, b) and full.shape == q.shape


def test_special_rows(bf, torch):  # noqa: F811
    batch = Batch(torch, [6], [6], 16)
    c = bf.PagedCache(8, 1, 16, 16)
    k = torch.randn(6, 1, 16, device="cuda")
    k[1, 0, 3], k[2, 0, 15], k[3] = float("nan"), float("inf"), 0.0
    pages = torch.zeros(batch.count, c.page_bytes, dtype=torch.uint8, device="cuda")
    q = c.append(pages, k, k, torch.ones_like(k), _frequencies(torch, 8), batch.d_tables, batch.d_lengths)
    back, values = c.read(pages, batch.d_tables, batch.d_lengths, 6)
    assert torch.isnan(back[1:3]).all() and torch.isfinite(back[[0, 3, 4, 5]]).all() and not back[3].any() and (values == 1).all()
    assert torch.isfinite(q[[0, 3, 4, 5]]).all() and torch.isnan(q[1, 0, [3, 11]]).all()


def test_going_back_raises_and_refusals(bf, torch):  # noqa: F811
    batch = Batch(torch, [6], [6], 16)
    c = bf.PagedCache(8, 2, 16, 16)
    pages = c.new_pages(batch.count)
    q, k, v = (torch.randn(6, 2, 16, device="cuda") for _ in range(3))
    f = _frequencies(torch, 8)
    rest = (batch.d_tables, batch.d_lengths)
    y = c.append(pages, q.clone().requires_grad_(True), k, v, f, *rest)
    assert torch.equal(y, c.append(pages, q, k, v, f, *rest))
    with pytest.raises(NotImplementedError):
        y.sum().backward()
    for args in ((q, k, v[:5], f), (q[:5], k, v, f), (q.half(), k, v, f), (q, k.half(), v, f), (q, k, v, f.double()), (q, k, v, f.cpu()), (q, k, v, f[None]),
                 (q[..., :8], k, v, f), (q, k[:, :1], v[:, :1], f)):
        with pytest.raises(ValueError):
            c.append(pages, *args, *rest)
    with pytest.raises(bf.BifeatError):
        c.append(pages, q, k, v, _frequencies(torch, 9), *rest)
    c.set_option("validate", 1)
    with pytest.raises(bf.BifeatError):
        c.append(pages, q, k, v, f, batch.d_tables, torch.tensor([1000], device="cuda"))
    assert c.append(pages, q, k, v, f, *rest) is not None


def test_going_back_to_frequencies_raises(bf, torch):  # noqa: F811
    batch = Batch(torch, [6], [6], 16)
    c = bf.PagedCache(8, 2, 16, 16)
    pages = c.new_pages(batch.count)
    q, k, v = (torch.randn(6, 2, 16, device="cuda") for _ in range(3))
    f = _frequencies(torch, 8)
    rest = (batch.d_tables, batch.d_lengths)
    y = c.append(pages, q, k, v, f.clone().requires_grad_(True), *rest)
    assert y.requires_grad and torch.equal(y, c.append(pages, q, k, v, f, *rest))
    with pytest.raises(NotImplementedError):
        y.sum().backward()
    assert c.append(pages, None, k, v, f.clone().requires_grad_(True), *rest) is None


def test_a_step_of_a_model_captured(bf, torch):  # noqa: F811
    """Product, turned keys, attention, product, routing, the experts' two products: together, and replayed."""
    heads, cached, d, width, E, top = 8, 2, 64, 256, 8, 2
    rng = np.random.default_rng(0)
    batch = Batch(torch, [40, 17, 33, 90], [1, 1, 1, 1], 16)
    w = lambda *shape: torch.from_numpy((rng.standard_normal(shape) / shape[-1] ** 0.5).astype(np.float32)).cuda()  # noqa: E731
    joint, back = bf.PackedLinear((heads + 2 * cached) * d, width), bf.PackedLinear(width, heads * d)
    up, down = bf.PackedLinear(384, width, experts=E), bf.PackedLinear(width, 384, experts=E)
    packed = [joint.pack(w(joint.out_features, width)), back.pack(w(width, heads * d)), up.pack(w(E, 384, width)), down.pack(w(E, width, 384))]
    router, f = w(width, E), _frequencies(torch, d // 2)
    c = bf.PagedCache(8, cached, d, 16)
    c.reserve()
    start = torch.from_numpy(_random_bytes(rng, batch.count, c.page_bytes)).cuda()
    c.write(start, *(torch.randn(180, cached, d, device="cuda").half() for _ in range(2)), batch.d_tables, batch.d_lengths,
            torch.tensor([0, 40, 57, 90, 180], device="cuda"))
    pages, x = start.clone(), torch.randn(4, width, device="cuda").half()

    def step():
        rows = joint.multiply(packed[0], x).view(4, heads + 2 * cached, d)
        q = c.append(pages, rows[:, :heads], rows[:, heads:heads + cached], rows[:, heads + cached:], f, batch.d_tables, batch.d_lengths)
        y = x + back.multiply(packed[1], c.attend(pages, q, batch.d_tables, batch.d_lengths).view(4, -1))
        ids, weights = bf.route(y.float() @ router, top)
        h = torch.relu(up.multiply_experts(packed[2], y, ids))
        return rows, q, ids, y + down.multiply_experts(packed[3], h, ids, weights)

    first = step()
    torch.cuda.synchronize()
    # the products against their weights in 32 bits: fp16 results (2^-11), sums of 16-bit rows in 32 bits
    want = x.float() @ joint.unpack(packed[0]).T
    assert (first[0].float().view(4, -1) - want).abs().max() <= 2.0 ** -10 * want.abs().max()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        x.copy_(torch.randn(4, width, device="cuda"))
        pages.copy_(start)
        want = step()
        torch.cuda.synchronize()
        held = pages.clone()
        pages.copy_(start)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and torch.equal(pages, held), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_angles_as_far_as_the_limit_and_past_it(bf, torch, dtype, interleaved):  # noqa: F811
    """Angles below 2^50 are turned by as any others; a pair whose angle is not gives NaN, and no number that looks like a key."""
    ps, far = 1024, 1 << 20
    batch = Batch(torch, [4], [4], ps)
    tables = torch.full((1, far // ps), -7, dtype=torch.int32, device="cuda")
    tables[0, -1] = 0
    batch.d_tables, batch.d_lengths, batch.lengths = tables, torch.tensor([far], device="cuda"), [far]
    batch.places = lambda: ((i, 0, (far - 4 + i) % ps) for i in range(4))
    f = torch.tensor([2.0 ** 30 - 64, 1.0, -2.0 ** 29, 2.0 ** 29 / 3, 12345678.0, 0.0, 2.0 ** -20, 3.5], device="cuda")   # (position times frequency: below 2^50)
    _check(bf, torch, batch, 8, 2, 2, 16, ps, dtype, "joint", 8, interleaved, frequencies=f)
    c = bf.PagedCache(8, 1, 16, ps)
    for bad in (2.0 ** 31, -2.0 ** 31, 2.0 ** 120, float("inf"), float("nan")):
        f[3] = bad
        k = torch.randn(4, 1, 16, device="cuda").to(_dtype(torch, dtype))
        pages = torch.zeros(1, c.page_bytes, dtype=torch.uint8, device="cuda")
        q = c.append(pages, k, k, k, f, batch.d_tables, batch.d_lengths, interleaved=interleaved)
        back, values = c.read(pages, batch.d_tables, batch.d_lengths, 4)
        nan = [6, 7] if interleaved else [3, 11]
        rest = [i for i in range(16) if i not in nan]
        assert torch.isnan(q[..., nan]).all() and torch.isfinite(q[..., rest]).all(), bad
        assert torch.isnan(back).all() and torch.isfinite(values).all(), bad
