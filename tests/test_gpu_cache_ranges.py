"""Attention over the paged cache at the ends of what it accepts, against its definition in 64 bits on what the pages hold: both kernels,
contexts that one workgroup has and that several share."""
import numpy as np
import pytest

import cache_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16", "bf16"]
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# relative rounding of a weight before it meets the values' codes
WEIGHT = {"f32": 2.0 ** -21, "f16": 2.0 ** -11, "bf16": 2.0 ** -11}
# new tokens, context, and whether the page table is far wider than it (which brings the kernel for many rows)
FORMS = {"few rows": (2, 300, False), "few rows, shared": (2, 1500, False), "many rows": (80, 120, False), "many rows, shared": (80, 700, True)}


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


def _decoded(raw, table, length, bits, heads, d, ps):
    """Keys and values [length, heads, d] in 64 bits, from the documented layout."""
    rb = ref.row_bytes(d, bits)
    blocks = raw[table].reshape(-1, heads, ps * (2 * rb + 16))
    with np.errstate(invalid="ignore"):   # (what no token was written to holds anything)
        floats = np.ascontiguousarray(blocks[:, :, 2 * ps * rb:]).view(np.float32).reshape(-1, heads, 4, ps).astype(np.float64)
    out = []
    for which in (0, 1):
        codes = blocks[:, :, which * ps * rb:(which + 1) * ps * rb].reshape(-1, heads, ps, rb)
        if bits == 4:
            codes = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:3], 2 * rb)
        with np.errstate(invalid="ignore"):
            x = floats[:, :, 2 * which + 1, :, None] + codes[..., :d].astype(np.float64) * floats[:, :, 2 * which, :, None]
        out.append(x.transpose(0, 2, 1, 3).reshape(-1, heads, d)[:length])
    return out


class Context:
    """One sequence of `length` cached tokens, the last n of which ask; keys and values [length, heads, d] in 32 bits."""

    def __init__(self, bf, torch, bits, keys, values, n, ps=64, wide=False):
        self.torch, self.bits, self.n, self.ps = torch, bits, n, ps
        self.length, self.heads, self.d = keys.shape
        self.c = bf.PagedCache(bits, self.heads, self.d, ps)
        held = -(-self.length // ps)
        table = np.random.default_rng(0).permutation(held + 2)[:held].astype(np.int32)
        self.tables = torch.full((1, 2 ** 20 // ps if wide else held), -7, dtype=torch.int32, device="cuda")
        self.tables[0, :held] = torch.from_numpy(table).cuda()
        self.lengths = torch.tensor([self.length], dtype=torch.int64, device="cuda")
        self.pages = self.c.new_pages(held + 2)
        self.c.write(self.pages, torch.from_numpy(keys.astype(np.float32)).cuda(), torch.from_numpy(values.astype(np.float32)).cuda(),
                     self.tables, self.lengths)
        self.keys, self.values = _decoded(self.pages.cpu().numpy(), table, self.length, bits, self.heads, self.d, ps)

    def check(self, q, dtype, scale=None, cap=0.0, scores=2.0 ** -19, weights=None):
        """q [n, query heads, d], rounded to dtype here; against the definition, to `scores` (of the largest sum of |q| |k|: products and sums in 32
        bits, which a weight and the weights' sum are off by) and `weights` (twice a weight's own rounding), both of the head's largest
        value, and the result's rounding."""
        torch, group = self.torch, q.shape[1] // self.heads
        scale = 1.0 / np.sqrt(self.d) if scale is None else scale
        weights = 2 * WEIGHT[dtype] if weights is None else weights
        tq = torch.from_numpy(q.astype(np.float32)).cuda().to(_dtype(torch, dtype))
        got = self.c.attend(self.pages, tq, self.tables, self.lengths, scale=scale, softcap=cap).float().cpu().numpy().astype(np.float64)
        hq = tq.float().cpu().numpy().astype(np.float64)
        # (the definition takes the softcap as a 32-bit number, as the entry point does)
        want = ref.attend(hq, self.keys, self.values, len(q), self.length, scale, float(np.float32(cap)))
        assert np.isfinite(got).all()
        live = max(0, len(q) - self.length)   # (the first of those that see something)
        for h in range(q.shape[1]):
            k, v = self.keys[:, h // group], self.values[:, h // group]
            biggest = (np.abs(hq[live:, h]) @ np.abs(k).T).max() * abs(scale)
            bound = np.abs(v).max() * (scores * biggest + weights) + HALF_ULP[dtype] * np.abs(want[:, h]) + (2.0 ** -25 if dtype == "f16" else 0)
            err = np.abs(got[:, h] - want[:, h])
            assert (err <= bound).all(), (h, (err / np.maximum(bound, 1e-300)).max(), np.argwhere(err > bound)[:3])
        return got, want


def _normal(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


# ------------------------------------------------------------------ values of any size

@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,constant", [("f16", 8192.0), ("f16", 60000.0), ("bf16", 1e7), ("f32", -1e7), ("bf16", 3e38), ("f32", 3e38), ("f32", 1e-20),
                                            ("f32", 1e-35), ("f16", 0.0)])
@pytest.mark.parametrize("bits,d,mixed", [(8, 64, False), (4, 1, False), (4, 100, True), (8, 256, True), (4, 128, False)])
def test_attend_over_value_rows_of_one_value(bf, torch, form, bits, d, mixed, dtype, constant):
    # rows whose columns are all alike have scale 0: all of a head's, or every other one beside ordinary rows
    n, m, wide = FORMS[form]
    values = np.full((m, 2, d), constant)
    if mixed:
        values[::2] = _normal(1, -(-m // 2), 2, d)
    if d > 1:
        values[:, 1] *= np.linspace(0.5, 1, m)[:, None]   # another value in each row of the second head
    context = Context(bf, torch, bits, _normal(2, m, 2, d), values, n, wide=wide)
    context.check(_normal(3, n, 4, d), dtype)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,size", [("bf16", 1e-25), ("f32", 1e-27), ("bf16", 1e-29), ("f32", 1e-29), ("f32", 1e-20), ("f32", 1e30), ("bf16", 1e37)])
@pytest.mark.parametrize("bits,d", [(8, 64), (4, 128), (8, 256)])
def test_attend_over_values_very_small_and_very_large(bf, torch, form, bits, d, dtype, size):
    n, m, wide = FORMS[form]
    context = Context(bf, torch, bits, _normal(2, m, 2, d), size * _normal(1, m, 2, d), n, wide=wide)
    # (weights of the smallest values are fp16 numbers below the normal ones: to 2^-9 and better)
    context.check(_normal(3, n, 4, d), dtype, weights=2 * max(WEIGHT[dtype], 2.0 ** -9) if size < 1e-28 else None)


# ------------------------------------------------------------------ caps of any size

@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("cap", [1e-38, 1e-30, 0.02, 5.0, 30.0, 50.0, 1e3, 1e4, 1e6, 1e9, 1e30, 3e38])
@pytest.mark.parametrize("dtype,bits,d", [("f32", 8, 64), ("f32", 4, 128), ("f16", 4, 64), ("bf16", 8, 256)])
def test_attend_with_caps_of_any_size(bf, torch, form, cap, dtype, bits, d):
    n, m, wide = FORMS[form]
    context = Context(bf, torch, bits, _normal(2, m, 2, d), _normal(1, m, 2, d), n, wide=wide)
    # scores of a standard deviation of 4; the cap's own error, a few 2^-24 of the score, is within what the sums are allowed
    context.check(4 * _normal(3, n, 4, d), dtype, cap=cap)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("cap", [0.0, 30.0, 50.0, 1e3])
@pytest.mark.parametrize("bits,d", [(8, 64), (4, 64), (8, 100), (4, 128), (8, 256)])
def test_32_bit_queries_keep_32_bits(bf, torch, form, cap, bits, d):
    # a query's pieces are off by 2^-23 of it, sums of products by a few 2^-24 of them, weights by 2^-23, in directions of their own: of scores of
    # a standard deviation of 2 that is below 2^-20 in the mean, and of the result no more than twice as much
    n, m, wide = FORMS[form]
    context = Context(bf, torch, bits, _normal(2, m, 2, d), _normal(1, m, 2, d), n, wide=wide)
    got, want = context.check(2 * _normal(3, n, 4, d), "f32", cap=cap)
    assert np.linalg.norm(got - want) <= 2.0 ** -19 * np.linalg.norm(want)


# ------------------------------------------------------------------ nothing to see

@pytest.mark.parametrize("d,n,ragged", [(64, 1, False), (256, 1, False), (128, 3, True), (64, 100, False), (256, 40, True)])
@pytest.mark.parametrize("dtype", TYPES)
def test_tables_without_room_leave_zeros(bf, torch, d, n, ragged, dtype):
    B, heads = 300, 8    # more items than run at a time
    c = bf.PagedCache(8, heads, d, 16)
    tables, lengths = torch.empty(B, 0, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int64, device="cuda")
    indptr = n * torch.arange(B + 1, device="cuda") if ragged else None
    out = torch.full((B * n, heads, d), 7.0, device="cuda", dtype=_dtype(torch, dtype))
    q = torch.randn(B * n, heads, d, device="cuda").to(out.dtype)
    pages = c.new_pages(1)
    c.attend(pages, q, tables, lengths, indptr, out=out)
    assert not out.any()
    c.write(pages, q, q, tables, lengths, indptr)
    assert not any(x.any() for x in c.read(pages, tables, lengths, B * n, indptr))


@pytest.mark.parametrize("n,m,wide", [(6, 3, False), (80, 70, True), (80, 70, False)])
@pytest.mark.parametrize("dtype,garbage", [("bf16", 1e30), ("f32", 1e30), ("f16", 65504.0), ("f32", 3e38), ("bf16", float("nan"))])
@pytest.mark.parametrize("bits,d", [(8, 64), (4, 100), (8, 256)])
def test_queries_before_the_beginning_may_hold_anything(bf, torch, n, m, wide, dtype, garbage, bits, d):
    context = Context(bf, torch, bits, _normal(2, m, 2, d), _normal(1, m, 2, d), n, wide=wide)
    q = _normal(3, n, 4, d)
    q[:n - m] = garbage
    with np.errstate(invalid="ignore"):
        got, _ = context.check(q, dtype)
    assert not got[:n - m].any()


def test_more_workgroups_than_a_launch_has_along_an_axis(bf, torch):
    # 2.1 million sequences of 8 heads, whose page tables have room for more units than are dealt: a workgroup each.  All look at the
    # same token, and answer with its values.
    B, heads, d, ps = 2 ** 21 + 3, 8, 8, 1024
    c = bf.PagedCache(8, heads, d, ps)
    tables = torch.zeros(B, 16, dtype=torch.int32, device="cuda")
    lengths = torch.ones(B, dtype=torch.int64, device="cuda")
    pages = c.new_pages(1)
    k = torch.randn(1, heads, d, device="cuda")
    c.write(pages, k, k, tables[:1], lengths[:1])
    values = c.read(pages, tables[:1], lengths[:1], 1, dtype=torch.bfloat16)[1]
    q = torch.randn(B, heads, d, device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, 9.0)
    c.attend(pages, q, tables, lengths, out=out)
    # a weight of 1 in one fp16 piece; the result's rounding
    assert (out - values).abs().max() <= 2.0 ** -7 * values.abs().max()


# ------------------------------------------------------------------ streams, threads, devices

def _two_contexts(bf, torch, c, n=2):
    """Two sequences of their own pages, queries, and what attending to them one after the other gives."""
    out = []
    for seed in (1, 2):
        tables = torch.from_numpy(np.random.default_rng(seed).permutation(80).astype(np.int32)[None]).cuda()
        lengths = torch.tensor([5000 + seed], dtype=torch.int64, device="cuda")
        pages = c.new_pages(80)
        k, v = (torch.from_numpy(_normal(10 * seed + i, 5000 + seed, c.heads, c.head_dim)).cuda().float() for i in (0, 1))
        c.write(pages, k, v, tables, lengths)
        q = torch.from_numpy(_normal(10 * seed + 2, n, 4 * c.heads, c.head_dim)).cuda().half()
        out.append((pages, q, tables, lengths, c.attend(pages, q, tables, lengths)))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("n", [2, 60])
def test_calls_of_one_object_on_two_streams_do_not_meet(bf, torch, n):
    # contexts that several workgroups share, whose parts are joined by a second kernel
    c = bf.PagedCache(8, 4, 64, 64)
    contexts = _two_contexts(bf, torch, c, n)
    streams = [torch.cuda.Stream() for _ in contexts]
    got = [[], []]
    for _ in range(40):
        for s, (pages, q, tables, lengths, _), g in zip(streams, contexts, got):
            with torch.cuda.stream(s):
                g.append(c.attend(pages, q, tables, lengths))
    torch.cuda.synchronize()
    for g, (*_, want) in zip(got, contexts):
        assert all(torch.equal(x, want) for x in g)


@pytest.mark.parametrize("shared", [False, True])
def test_threads_share_an_object(bf, torch, shared):
    import threading
    c = bf.PagedCache(8, 4, 64, 64)
    contexts = _two_contexts(bf, torch, c)
    fresh, wrong = bf.PagedCache(8, 4, 64, 64), []
    one = torch.cuda.Stream()

    def run(pages, q, tables, lengths, want):
        with torch.cuda.stream(one if shared else torch.cuda.Stream()):
            got = [fresh.attend(pages, q, tables, lengths) for _ in range(100)]
            torch.cuda.current_stream().synchronize()
            wrong.extend(i for i, x in enumerate(got) if not torch.equal(x, want))

    threads = [threading.Thread(target=run, args=x) for x in contexts]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not wrong and not any(t.is_alive() for t in threads)


def test_a_replayed_graph_and_other_calls_do_not_meet(bf, torch):
    c = bf.PagedCache(8, 4, 64, 64)
    (pages, q, tables, lengths, want), (pages2, q2, tables2, lengths2, want2) = _two_contexts(bf, torch, c)
    out, graph = torch.zeros_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(pages, q, tables, lengths, out=out)
    side = torch.cuda.Stream()
    for _ in range(20):
        out.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        got = [c.attend(pages2, q2, tables2, lengths2) for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(torch.equal(x, want2) for x in got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits,d", [(8, 64), (4, 128), (8, 256)])
def test_captured_calls_of_many_rows_without_a_workspace(bf, torch, bits, d, dtype):
    # nothing is split: the kernel for many rows with an item a workgroup, over a table far wider than the context
    context = Context(bf, torch, bits, _normal(2, 300, 2, d), _normal(1, 300, 2, d), 80, wide=True)
    fresh, eager = bf.PagedCache(bits, 2, d, 64), context.c
    q, out, graph = torch.zeros(80, 4, d, dtype=_dtype(torch, dtype), device="cuda"), None, torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fresh.attend(context.pages, q, context.tables, context.lengths)

    class Replayed:
        def attend(self, pages, now, *args, **kw):
            q.copy_(now)
            out.zero_()
            graph.replay()
            return out

    for seed in range(3):
        x = _normal(seed, 80, 4, d)
        context.c = Replayed()
        context.check(x, dtype)
        context.c = eager
        context.check(x, dtype)


def test_branches_of_a_graph_do_not_meet(bf, torch):
    c = bf.PagedCache(8, 4, 64, 64)
    contexts = _two_contexts(bf, torch, c)
    outs, graph, side = [torch.zeros_like(x[1]) for x in contexts], torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        for stream, (pages, q, tables, lengths, _), out in zip((main, side), contexts, outs):
            with torch.cuda.stream(stream):
                c.attend(pages, q, tables, lengths, out=out)
        main.wait_stream(side)
    for _ in range(10):
        for x, out in zip(contexts, outs):
            x[1].copy_(torch.randn_like(x[1]))
            out.zero_()
        graph.replay()
        wants = [c.attend(*x[:4]) for x in contexts]
        torch.cuda.synchronize()
        assert torch.equal(outs[0], wants[0])
        # the second branch has no workspace, so that its context is not split: other sums; fp16's rounding of each, and of values below 4
        assert (outs[1].float() - wants[1].float()).abs().max() <= 2 * 2.0 ** -11 * 4


def test_tensors_of_another_device_are_refused(bf, torch, monkeypatch):
    c = bf.PagedCache(8, 2, 64, 16)
    pages, x = c.new_pages(2), torch.zeros(1, 2, 64, device="cuda")
    tables, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int64, device="cuda")
    calls = [lambda: c.write(pages, x, x, tables, lengths), lambda: c.read(pages, tables, lengths, 1),
             lambda: c.attend(pages, x, tables, lengths), lambda: c.check(pages, tables, lengths)]
    for call in calls:
        call()
    for call in [lambda: c.write(pages, x, x, tables.cpu(), lengths), lambda: c.attend(pages, x, tables, lengths.cpu()),
                 lambda: c.attend(pages.cpu(), x, tables, lengths), lambda: c.read(pages.cpu(), tables, lengths, 1)]:
        with pytest.raises(ValueError):
            call()
    # the pages' device is not the current one (behind the native module, which asks for it itself)
    import paper_2207_14696_amd.binding as binding
    monkeypatch.setattr(binding, "_calls", False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("native", [True, False])
def test_attend_does_not_drop_a_gradient_silently(bf, torch, monkeypatch, native):
    if not native:
        import paper_2207_14696_amd.binding as binding
        monkeypatch.setattr(binding, "_calls", False)
    context = Context(bf, torch, 8, _normal(1, 40, 2, 64), _normal(2, 40, 2, 64), 3)
    q = torch.from_numpy(_normal(3, 3, 4, 64)).float().cuda().requires_grad_()
    args = (context.tables, context.lengths)
    got = context.c.attend(context.pages, q, *args, window=20)
    with torch.no_grad():
        want = context.c.attend(context.pages, q, *args, window=20)
    assert torch.equal(got, want) and got.requires_grad and not want.requires_grad
    with pytest.raises(NotImplementedError):
        got.sum().backward()
    with pytest.raises(ValueError):
        context.c.attend(context.pages, q, *args, out=torch.empty_like(want))
    assert not context.c.attend(context.pages, q.detach(), *args).requires_grad


# ------------------------------------------------------------------ large sums of products

@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("bits,d", [(4, 64), (4, 128), (4, 256), (8, 64), (8, 128), (8, 256)])
def test_scores_of_large_sums(bf, torch, bits, d, many):
    """Two positions whose scores are nearly alike, of products that add up to tens of thousands: their weights' ratio shows the difference."""
    rng, scale, n, ps = np.random.default_rng(d + bits), 256.0, 8192, 16
    c = bf.PagedCache(bits, 1, d, ps)

    def cached(keys, tables, lengths):
        """The keys in the cache, as they stand there, beside values (1, 0, 0, ..), (0, 1, 0, ..), (1, 0, ..), .."""
        k = torch.from_numpy(keys[:, None]).float().cuda()
        v = torch.zeros_like(k)
        v[0::2, :, 0], v[1::2, :, 1] = 1, 1
        pages = c.new_pages(int(tables.max()) + 1)
        c.write(pages, k, v, tables, lengths)
        return pages, c.read(pages, tables, lengths, len(k))[0].double().cpu().numpy()[:, 0]

    q = rng.standard_normal(d).astype(np.float16).astype(np.float64)
    keys = rng.standard_normal((n, d))
    _, stand = cached(keys, torch.arange(n // ps, dtype=torch.int32, device="cuda")[None], torch.tensor([n], device="cuda"))
    pairs = np.argsort(stand @ q).reshape(-1, 2)[::4]
    B, group, last = len(pairs), 40 if many else 1, 2 if many else 1
    tables = torch.zeros(B, 2 ** 20 // ps if many else 1, dtype=torch.int32, device="cuda")
    tables[:, 0] = torch.arange(B, device="cuda")
    lengths = torch.full((B,), 2, dtype=torch.int64, device="cuda")
    pages, k = cached(keys[pairs.reshape(-1)], tables, lengths)
    k = k.reshape(B, 2, d)
    tq = torch.from_numpy(q).half().cuda().expand(last * B, group, d)
    out = c.attend(pages, tq, tables, lengths, scale=scale).double().cpu().numpy().reshape(B, last, group, d)[:, -1]
    away = scale * (k[:, 0] - k[:, 1]) @ q
    seen = np.abs(away) < 1
    assert seen.sum() > 50
    got = np.log(out[seen, :, 0] / out[seen, :, 1])
    # Sums of products in 32 bits: 2^-22 of the sum of their sizes.  A weight is off by 2^-12 of it, which meets half its row's range, 1/2, in both
    # columns: 2^-13 of their weights' sum 1 in each of two outputs of 1 / (1 + e) or more, 3.8 2^-11 in all; and the two results' 2^-11.
    bound = 2.0 ** -22 * scale * (np.abs(k) @ np.abs(q)).max(-1)[seen] + 6 * 2.0 ** -11
    err = np.abs(got - away[seen, None]).max(-1)
    assert (err <= bound).all(), (err / bound).max()
