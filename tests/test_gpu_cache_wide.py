"""Attention over the paged cache with page tables far wider than the contexts: the kernel for many rows, which short contexts
take only then, does what the other does, at the same sizes and masks.  And rows read back past the caches."""
import numpy as np
import pytest

import test_gpu_cache as base
from test_gpu_cache import SHAPES, TYPES, bf, torch  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def wide(monkeypatch):
    class Wide(base.Batch):
        def __init__(self, torch, lengths, news, ps, *args, **more):
            super().__init__(torch, lengths, news, ps, *args, **more)
            narrow = self.d_tables
            self.d_tables = torch.full((len(lengths), 2 ** 20 // ps), -7, dtype=torch.int32, device="cuda")
            self.d_tables[:, :narrow.shape[1]] = narrow
    monkeypatch.setattr(base, "Batch", Wide)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_attend_of_chunks(bf, torch, shape, dtype):  # noqa: F811
    bits, heads, group, d, ps = shape
    more = 64 // group  # (rows enough for that kernel, whatever the group)
    base._attend_case(bf, torch, bits, heads, group, d, ps, dtype, [70, 150, 90, 33, 5, 0, 129 + more * 7],
                      [70, 40, 1, 0, 8, 3, 129 + more * 7])


@pytest.mark.parametrize("opts", [
    dict(window=1), dict(window=17), dict(window=64, prefix=[5, 0, 200, 64]), dict(window=33, slopes=True), dict(prefix=[0, 70, 41, 300]),
    dict(cap=5.0), dict(cap=30.0, slopes=True, window=100), dict(slopes=True), dict(scale=0.5), dict(scale=-0.3), dict(scale=0.0)])
@pytest.mark.parametrize("dtype,bits,group,d", [("f16", 8, 4, 128), ("bf16", 4, 2, 64), ("f32", 4, 3, 100), ("bf16", 8, 2, 256)])
def test_attend_with_every_mask(bf, torch, opts, dtype, bits, group, d):  # noqa: F811
    base._attend_case(bf, torch, bits, 2, group, d, 16, dtype, [100, 260, 41, 130], [100, 20, 1, 130], **opts)


@pytest.mark.parametrize("layout", ["packed", "joint", "heads_first", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,news", [(64, [50, 3, 70]), (33, [60, 3, 70]), (130, [60, 3, 70])])
def test_attend_to_queries_in_any_layout(bf, torch, layout, dtype, d, news):  # noqa: F811
    base._attend_case(bf, torch, 8, 2, 2, d, 32, dtype, [60, 100, 200], news, layout=layout)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [[1, 1], [90, 60]])
def test_attend_over_values_of_very_different_sizes(bf, torch, dtype, news):  # noqa: F811
    base._attend_case(bf, torch, 8, 2, 2, 64, 16, dtype, [600, 90], news, spread=3.0, q_scale=4.0)


@pytest.mark.parametrize("news", [[1, 1, 1], [300, 5, 1]])
@pytest.mark.parametrize("bits,d,group", [(8, 128, 4), (4, 64, 1), (4, 256, 2)])
def test_attend_over_long_contexts(bf, torch, news, bits, d, group):  # noqa: F811
    base._attend_case(bf, torch, bits, 1, group, d, 64, "f16", [6001, 40, 2999], news, seed=5)


@pytest.mark.parametrize("opts", [dict(window=300, prefix=[130, 700]), dict(window=64, slopes=True), dict(window=1000, prefix=[1, 0], cap=20.0)])
@pytest.mark.parametrize("dtype,bits,d", [("f16", 4, 64), ("bf16", 8, 256), ("f32", 8, 128)])
def test_attend_over_a_window_and_a_prefix_far_apart(bf, torch, opts, dtype, bits, d):  # noqa: F811
    base._attend_case(bf, torch, bits, 2, 2, d, 64, dtype, [1500, 900], [200, 90], **opts)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_a_query_does_not_see_does_not_reach_it(bf, torch, dtype):  # noqa: F811
    base.test_what_a_query_does_not_see_does_not_reach_it(bf, torch, 100, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_query_that_is_not_finite_spoils_itself_only(bf, torch, dtype):  # noqa: F811
    base.test_a_query_that_is_not_finite_spoils_itself_only(bf, torch, dtype, 40)


@pytest.mark.parametrize("bits,dtype,d", [(8, "bf16", 128), (4, "f16", 64), (8, "f32", 100)])
def test_a_prompt_and_its_answer_in_steps(bf, torch, bits, dtype, d):  # noqa: F811
    base.test_a_prompt_and_its_answer_in_steps(bf, torch, bits, dtype, d)


@pytest.mark.parametrize("heads,n,d", [(1, 1, 64), (2, 1, 128), (1, 3, 256), (16, 1, 64), (8, 40, 128)])
def test_one_context_of_many_parts(bf, torch, heads, n, d):  # noqa: F811
    # an item of many workgroups' parts, and of few (the joins' two forms), the same as twice as many queries in one call
    c, ps, m = bf.PagedCache(8, heads, d, 64), 64, 20000
    rng = np.random.default_rng(2)
    tables = torch.from_numpy(rng.permutation(m // ps + 1).astype(np.int32)[None]).cuda()
    pages = c.new_pages(m // ps + 1)
    k, v, q = (base._rows(torch, rng, m if h == heads else n, h, d, "bf16", "packed") for h in (heads, heads, 2 * heads))
    lengths = torch.tensor([m], dtype=torch.int64, device="cuda")
    c.write(pages, k, v, tables, lengths)
    got = c.attend(pages, q, tables, lengths).double().cpu()
    keys, values = (x.double().cpu() for x in c.read(pages, tables, lengths, m))
    s = torch.einsum("nhgd,mhd->nhgm", q.double().cpu().view(n, heads, 2, d), keys) / d ** 0.5
    seen = torch.arange(m)[None] <= torch.arange(m - n, m)[:, None]
    w = s.masked_fill(~seen[:, None, None], -torch.inf).softmax(-1)
    want = torch.einsum("nhgm,mhd->nhgd", w, values).reshape(n, 2 * heads, d)
    # scores' products in 32 bits, the weight's rounding twice, the result's
    biggest = (q.double().abs().amax().item() * keys.abs().sum(-1).amax().item()) / d ** 0.5
    bound = values.abs().max() * (2 * 2.0 ** -20 * biggest + 2 * 2.0 ** -11) + 2.0 ** -8 * want.abs() + 2.0 ** -25
    assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits,heads,d", [(8, 3, 100), (4, 2, 128), (4, 5, 37), (8, 1, 256), (8, 4, 6)])
def test_large_reads_are_small_ones_together(bf, torch, bits, heads, d, dtype):  # noqa: F811
    n, ps = (40 << 20) // (8 * heads * d) + 5, 64   # past 16 MB in any type
    c = bf.PagedCache(bits, heads, d, ps)
    tables = torch.randperm(-(-n // ps), device="cuda").to(torch.int32)[None].contiguous()
    pages = c.new_pages(tables.numel())
    k, v = (torch.randn(n, heads, d, device="cuda") for _ in range(2))
    lengths = torch.tensor([n], dtype=torch.int64, device="cuda")
    c.write(pages, k, v, tables, lengths)
    got = c.read(pages, tables, lengths, n, dtype=base._dtype(torch, dtype))
    for end in (333, n // 3, n):
        part = c.read(pages, tables, torch.tensor([end], dtype=torch.int64, device="cuda"), 333, dtype=base._dtype(torch, dtype))
        for whole, some in zip(got, part):
            assert torch.equal(whole[end - 333:end], some)
