"""The paged cache on the GPU against its definition in 64 bits: codes bit for bit, values read back, attention of
single tokens and of chunks, every mask, and what lies outside the masks."""
import numpy as np
import pytest

import cache_reference as ref

pytestmark = pytest.mark.gpu

TYPES = ["f32", "f16", "bf16"]
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
# relative rounding of a weight before it meets the values' codes: fp16 to nearest, or two such pieces
WEIGHT = {"f32": 2.0 ** -21, "f16": 2.0 ** -11, "bf16": 2.0 ** -11}


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
    """A tensor's values, exactly."""
    return t.detach().float().cpu().numpy()


class Batch:
    """Sequences whose pages lie anywhere among pages of arbitrary bytes."""

    def __init__(self, torch, lengths, news, ps, seed=0, spare=3):
        rng = np.random.default_rng(seed)
        self.lengths, self.news, self.ps = list(lengths), list(news), ps
        B, self.width = len(lengths), max([-(-m // ps) for m in lengths] + [1])
        self.count = B * self.width + spare
        self.tables = rng.permutation(self.count)[:B * self.width].reshape(B, self.width).astype(np.int32)
        self.starts = np.concatenate([[0], np.cumsum(news)]).astype(np.int64)
        self.T = int(self.starts[-1])
        # entries past a sequence's last page are not looked at
        shown = self.tables.copy()
        for b, m in enumerate(lengths):
            shown[b, -(-m // ps):] = -7
        self.d_tables = torch.from_numpy(shown).cuda()
        self.d_lengths = torch.tensor(self.lengths, dtype=torch.int64, device="cuda")
        self.d_indptr = torch.from_numpy(self.starts).cuda()

    def places(self):
        """(token, page, slot) of every token of the call that has a place."""
        for b, (m, n) in enumerate(zip(self.lengths, self.news)):
            for i in range(n):
                p = m - n + i
                if p >= 0:
                    yield int(self.starts[b]) + i, int(self.tables[b, p // self.ps]), p % self.ps


def _random_bytes(rng, count, page_bytes):
    return rng.integers(0, 256, (count, page_bytes), dtype=np.uint8)


def _rows(torch, rng, T, heads, d, dtype, layout="joint", scale=1.0):
    """[T, heads, d] in one of the layouts that models have."""
    x = torch.from_numpy((scale * rng.standard_normal((T, heads, d))).astype(np.float32)).cuda().to(_dtype(torch, dtype))
    if layout == "packed":
        return x
    if layout == "joint":      # a slice of a joint projection that begins anywhere
        wide = torch.empty(T, heads + 3, d, dtype=x.dtype, device="cuda")
        wide[:, 1:heads + 1] = x
        return wide[:, 1:heads + 1]
    if layout == "heads_first":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "odd":        # rows an odd number of elements apart
        wide = torch.empty(T * (heads * (d + 1) + 1) + 1, dtype=x.dtype, device="cuda")
        view = torch.as_strided(wide, (T, heads, d), (heads * (d + 1) + 1, d + 1, 1), 1)
        view.copy_(x)
        return view
    raise ValueError(layout)


def _filled(torch, batch, c, bits, heads, d, seed, spread=1.0, dtype="f32"):
    """Pages that hold every sequence as a whole, by the definition; what was never written is arbitrary, its floats NaN."""
    rng = np.random.default_rng(seed)
    raw = _random_bytes(rng, batch.count, c.page_bytes)
    pages = ref.Pages(raw, bits, heads, d, batch.ps)
    raw.reshape(batch.count, heads, -1)[:, :, 2 * batch.ps * pages.rb:] = 0xff
    column = np.exp(0.5 * rng.standard_normal((heads, d)))
    middle = 0.5 * rng.standard_normal((heads, d))
    for b, m in enumerate(batch.lengths):
        for j in range(m):
            page, slot = int(batch.tables[b, j // batch.ps]), j % batch.ps
            k = middle + column * rng.standard_normal((heads, d))
            v = np.exp(spread * rng.standard_normal((heads, 1))) * rng.standard_normal((heads, d))
            for h in range(heads):
                pages.put(page, slot, h, 0, k[h])
                pages.put(page, slot, h, 1, v[h])
    return raw, pages


# ------------------------------------------------------------------ write

@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,heads,d,ps,layout", [
    ("f16", 12, 64, 16, "joint"), ("bf16", 8, 128, 64, "packed"), ("f32", 2, 100, 16, "odd"), ("f16", 1, 256, 32, "heads_first"),
    ("bf16", 3, 37, 16, "odd"), ("f32", 5, 1, 16, "packed"), ("f16", 7, 129, 128, "odd"), ("bf16", 2, 8, 1024, "heads_first")])
def test_write_matches_the_definition_bit_for_bit(bf, torch, bits, dtype, heads, d, ps, layout):
    rng = np.random.default_rng(d + bits)
    # one token, a page's edge, several pages, none, more tokens than places, a token that begins a page
    batch = Batch(torch, [1, ps, 2 * ps + 5, 40, 3, ps + 1], [1, 3, ps + 7, 0, 5, 1], ps)
    c = bf.PagedCache(bits, heads, d, ps)
    want = _random_bytes(rng, batch.count, c.page_bytes)
    pages = torch.from_numpy(want.copy()).cuda()
    k, v = (_rows(torch, rng, batch.T, heads, d, dtype, layout) for _ in range(2))
    c.write(pages, k, v, batch.d_tables, batch.d_lengths, batch.d_indptr)
    oracle = ref.Pages(want, bits, heads, d, ps)
    hk, hv = _host(k), _host(v)
    for t, page, slot in batch.places():
        for h in range(heads):
            oracle.put(page, slot, h, 0, hk[t, h])
            oracle.put(page, slot, h, 1, hv[t, h])
    got = pages.cpu().numpy()
    assert np.array_equal(got, want), f"{(got != want).sum()} bytes differ"


@pytest.mark.parametrize("bits", [4, 8])
def test_write_of_special_rows(bf, torch, bits):
    heads, d, ps = 1, 24, 16
    rows = np.tile(np.linspace(-1, 2, d, dtype=np.float32), (12, 1))
    rows[1] = 3.25                      # all alike
    rows[2] = 0.0
    rows[3] = -0.0
    rows[4, 5] = np.nan
    rows[5, 0] = np.inf
    rows[6, 23] = -np.inf
    rows[7] = np.linspace(-3e38, 3e38, d)          # the range overflows
    rows[8] = np.linspace(0, 1e-39, d)              # too narrow for a reciprocal
    rows[9] = 1e-30 * np.linspace(-1, 2, d)
    rows[10] = 1e37 * np.linspace(-1, 2, d)
    rows[11] = np.where(np.arange(d) % 2, 1.0, np.nextafter(np.float32(1), np.float32(2)))
    batch = Batch(torch, [12], [12], ps)
    c = bf.PagedCache(bits, heads, d, ps)
    want = _random_bytes(np.random.default_rng(0), batch.count, c.page_bytes)
    pages = torch.from_numpy(want.copy()).cuda()
    x = torch.from_numpy(rows[:, None, :]).cuda()
    c.write(pages, x, x, batch.d_tables, batch.d_lengths)
    oracle = ref.Pages(want, bits, heads, d, ps)
    for t, page, slot in batch.places():
        oracle.put(page, slot, 0, 0, rows[t])
        oracle.put(page, slot, 0, 1, rows[t])
    got = ref.Pages(pages.cpu().numpy(), bits, heads, d, ps)
    for t, page, slot in batch.places():
        for which in (0, 1):
            assert np.array_equal(got.codes(page, 0, which, slot), oracle.codes(page, 0, which, slot)), t
            for i in (2 * which, 2 * which + 1):
                assert np.array_equal(got.float_at(page, 0, i, slot), oracle.float_at(page, 0, i, slot), equal_nan=True), t
    k, v = c.read(pages, batch.d_tables, batch.d_lengths, 12)
    k = k.cpu().numpy()[:, 0]
    assert np.isnan(k[4:8]).all() and np.isfinite(k[[0, 1, 2, 3, 8, 9, 10, 11]]).all()
    assert (k[1] == 3.25).all() and not k[2:4].any()
    span = rows.max(-1) - rows.min(-1)
    for t in (0, 9, 10, 11):
        # half a level, and the roundings of range, reciprocal, product and level: a few 2^-24 of the largest
        assert np.abs(k[t] - rows[t]).max() <= span[t] / (2 * ((1 << bits) - 1)) + 2.0 ** -21 * np.abs(rows[t]).max()


# ------------------------------------------------------------------ read

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits,heads,d,ps", [(8, 12, 64, 16), (4, 8, 128, 64), (4, 2, 100, 16), (8, 1, 256, 32), (4, 3, 37, 16), (8, 2, 1, 16)])
def test_read_gives_the_values_that_the_codes_stand_for(bf, torch, dtype, bits, heads, d, ps):
    batch = Batch(torch, [1, ps, 2 * ps + 5, 40, 3, 0], [1, ps, 7, 0, 5, 2], ps, seed=d)
    c = bf.PagedCache(bits, heads, d, ps)
    raw, pages = _filled(torch, batch, c, bits, heads, d, seed=d + 1)
    got = c.read(torch.from_numpy(raw).cuda(), batch.d_tables, batch.d_lengths, batch.T, batch.d_indptr, dtype=_dtype(torch, dtype))
    want = np.zeros((2, batch.T, heads, d))
    size = np.zeros((2, batch.T, heads, 1))
    for t, page, slot in batch.places():
        for which in (0, 1):
            for h in range(heads):
                want[which, t, h] = pages.get(page, slot, h, which)
                size[which, t, h] = abs(pages.float_at(page, h, 2 * which + 1, slot)[0]) + abs(want[which, t, h]).max()
    for which in (0, 1):
        x = _host(got[which]).astype(np.float64)
        # one rounding of the sum in 32 bits, one to the type (its subnormals: 2^-25)
        bound = 2.0 ** -23 * size[which] + HALF_ULP[dtype] * np.abs(want[which]) + 2.0 ** -25
        assert (np.abs(x - want[which]) <= bound).all()
        assert not x[batch.starts[4]:batch.starts[4] + 2].any() and not x[batch.starts[5]:].any()   # before the beginning


def test_read_into_given_arrays_and_by_default(bf, torch):
    batch = Batch(torch, [20, 33], [20, 20], 16)
    c = bf.PagedCache(8, 2, 64, 16)
    raw, _ = _filled(torch, batch, c, 8, 2, 64, seed=0)
    pages = torch.from_numpy(raw).cuda()
    k, v = c.read(pages, batch.d_tables, batch.d_lengths, 40)
    assert k.dtype == v.dtype == torch.float32
    out = (torch.full_like(k, 9), torch.full_like(v, 9))
    assert c.read(pages, batch.d_tables, batch.d_lengths, 40, batch.d_indptr, out=out)[0] is out[0]
    assert torch.equal(out[0], k) and torch.equal(out[1], v)


# ------------------------------------------------------------------ attend

def _attend_case(bf, torch, bits, heads, group, d, ps, dtype, lengths, news, scale=None, cap=0.0, window=0, prefix=None, slopes=False,
                 layout="joint", uniform=False, seed=0, spread=1.0, q_scale=1.0):
    rng = np.random.default_rng(seed + 17)
    batch = Batch(torch, lengths, news, ps, seed)
    c = bf.PagedCache(bits, heads, d, ps)
    raw, pages = _filled(torch, batch, c, bits, heads, d, seed + 1, spread)
    q = _rows(torch, rng, batch.T, heads * group, d, dtype, layout, q_scale)
    sl = 2.0 ** (-8.0 * np.arange(1, heads * group + 1) / (heads * group)) if slopes else None
    out = c.attend(torch.from_numpy(raw).cuda(), q, batch.d_tables, batch.d_lengths, None if uniform else batch.d_indptr, scale=scale,
                   softcap=cap, window=window, prefix=None if prefix is None else torch.tensor(prefix, dtype=torch.int64, device="cuda"),
                   slopes=None if sl is None else torch.from_numpy(sl.astype(np.float32)).cuda())
    assert out.dtype == q.dtype and out.shape == q.shape
    got, hq = _host(out).astype(np.float64), _host(q).astype(np.float64)
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    for b, (m, n) in enumerate(zip(lengths, news)):
        part = slice(int(batch.starts[b]), int(batch.starts[b + 1]))
        keys, values = (pages.sequence(batch.tables[b], m, w) for w in (0, 1))
        want = ref.attend(hq[part], keys, values, n, m, scale, cap, window, 0 if prefix is None else prefix[b], sl)
        if n == 0:
            continue
        # products and sums in 32 bits: 2^-20 of the largest sum of products and of the bias, which twice over is what a
        # weight and the weights' sum can be off by; then the weight's own rounding (and as much again for the 32-bit
        # sums of weights and values), and the result's
        biggest = 0.0
        for h in range(heads * group):
            if m:
                biggest = max(biggest, (np.abs(hq[part][:, h]) @ np.abs(keys[:, h // group]).T).max() * abs(scale))
        biggest += m * (sl.max() if slopes else 0.0)
        top = np.abs(values).max() if m else 0.0
        bound = top * (2 * 2.0 ** -20 * biggest + 2 * WEIGHT[dtype]) + HALF_ULP[dtype] * np.abs(want) + 2.0 ** -25
        err = np.abs(got[part] - want)
        assert (err <= bound).all(), (b, (err / bound).max(), np.argwhere(err > bound)[:3])
    return got


SHAPES = [  # bits, heads, group, d, page
    (8, 2, 4, 128, 64), (4, 2, 4, 128, 16), (8, 3, 1, 64, 16), (4, 1, 8, 64, 32), (8, 1, 5, 256, 32), (4, 2, 2, 256, 128),
    (4, 2, 5, 100, 16), (8, 2, 3, 80, 16), (8, 1, 1, 37, 16), (4, 1, 2, 1, 16), (4, 1, 17, 96, 64), (8, 1, 33, 33, 16), (4, 1, 3, 255, 1024)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_attend_of_single_tokens(bf, torch, shape, dtype):
    bits, heads, group, d, ps = shape
    lengths = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 130, 257]
    _attend_case(bf, torch, bits, heads, group, d, ps, dtype, lengths, [1] * len(lengths), uniform=True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_attend_of_chunks(bf, torch, shape, dtype):
    bits, heads, group, d, ps = shape
    # a whole prompt, a chunk behind a context, a single token, none, more queries than the sequence has tokens, no sequence
    _attend_case(bf, torch, bits, heads, group, d, ps, dtype, [70, 150, 90, 33, 5, 0, 129], [70, 40, 1, 0, 8, 3, 129])


@pytest.mark.parametrize("opts", [
    dict(window=1), dict(window=17), dict(window=64, prefix=[5, 0, 200, 64]), dict(window=33, slopes=True), dict(prefix=[0, 70, 41, 300]),
    dict(cap=5.0), dict(cap=30.0, slopes=True, window=100), dict(slopes=True), dict(scale=0.5), dict(scale=-0.3), dict(scale=0.0)])
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [3, 3, 3, 3], [100, 20, 1, 130]])
@pytest.mark.parametrize("dtype,bits,group,d", [("f16", 8, 4, 128), ("bf16", 4, 2, 64), ("f32", 4, 3, 100)])
def test_attend_with_every_mask(bf, torch, opts, news, dtype, bits, group, d):
    _attend_case(bf, torch, bits, 2, group, d, 16, dtype, [100, 260, 41, 130], news, **opts)


@pytest.mark.parametrize("layout", ["packed", "joint", "heads_first", "odd"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,news", [(64, [2, 2, 2]), (64, [50, 3, 70]), (33, [1, 1, 1]), (33, [60, 3, 70])])
def test_attend_to_queries_in_any_layout(bf, torch, layout, dtype, d, news):
    _attend_case(bf, torch, 8, 2, 2, d, 32, dtype, [60, 100, 200], news, layout=layout)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [[1, 1], [90, 60]])
def test_attend_over_values_of_very_different_sizes(bf, torch, dtype, news):
    # values' sizes over e^+-9, queries that pick single positions
    _attend_case(bf, torch, 8, 2, 2, 64, 16, dtype, [600, 90], news, spread=3.0, q_scale=4.0)


@pytest.mark.parametrize("news", [[1, 1, 1], [16, 16, 16], [300, 5, 1]])
@pytest.mark.parametrize("bits,d,group", [(8, 128, 4), (4, 64, 1), (4, 256, 2)])
def test_attend_over_long_contexts(bf, torch, news, bits, d, group):
    # contexts that several workgroups share, beside short ones
    _attend_case(bf, torch, bits, 1, group, d, 64, "f16", [6001, 40, 2999], news, seed=5)


def test_attend_sums_are_the_same_every_time(bf, torch):
    a = _attend_case(bf, torch, 8, 2, 4, 64, 16, "f32", [3000, 100], [1, 1])
    b = _attend_case(bf, torch, 8, 2, 4, 64, 16, "f32", [3000, 100], [1, 1])
    assert np.array_equal(a, b)


@pytest.mark.parametrize("n", [4, 100])
@pytest.mark.parametrize("dtype", TYPES)
def test_what_a_query_does_not_see_does_not_reach_it(bf, torch, n, dtype):
    heads, group, d, ps, m = 2, 2, 64, 16, 150
    batch = Batch(torch, [m], [n], ps)
    c = bf.PagedCache(8, heads, d, ps)
    raw, _ = _filled(torch, batch, c, 8, heads, d, seed=3)
    pages = torch.from_numpy(raw).cuda()
    rng = np.random.default_rng(4)
    q = _rows(torch, rng, n, heads * group, d, dtype)
    clean = c.attend(pages, q, batch.d_tables, batch.d_lengths)
    # the last token but one of the call, and one far back, hold NaN and infinity
    one = Batch(torch, [m - 1], [1], ps)
    one.d_tables = batch.d_tables
    bad = _rows(torch, rng, 1, heads, d, "f32", "packed")
    bad[0, 0, 3], bad[0, 1, 5] = float("nan"), float("inf")
    c.write(pages, bad, bad, one.d_tables, one.d_lengths)
    got = c.attend(pages, q, batch.d_tables, batch.d_lengths)
    assert torch.equal(got[:n - 2], clean[:n - 2])
    assert got[n - 2:].isnan().all()
    # outside the window it is not seen either
    old = Batch(torch, [20], [1], ps)
    c.write(pages, bad, bad, batch.d_tables, old.d_lengths)
    pages2 = torch.from_numpy(raw).cuda()
    c.write(pages2, bad, bad, batch.d_tables, old.d_lengths)
    w = m - n - 20 + 1   # the first query's window begins at position 20
    seen = c.attend(pages2, q, batch.d_tables, batch.d_lengths, window=w)
    want = c.attend(torch.from_numpy(raw).cuda(), q, batch.d_tables, batch.d_lengths, window=w)
    assert torch.equal(seen, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 40])
def test_a_query_that_is_not_finite_spoils_itself_only(bf, torch, dtype, n):
    batch = Batch(torch, [90], [n], 16)
    c = bf.PagedCache(8, 1, 64, 16)
    raw, _ = _filled(torch, batch, c, 8, 1, 64, seed=3)
    pages = torch.from_numpy(raw).cuda()
    q = _rows(torch, np.random.default_rng(1), n, 4, 64, dtype, "packed")
    clean = c.attend(pages, q, batch.d_tables, batch.d_lengths)
    q[0, 1, 7], q[0, 2, 60] = float("nan"), float("inf")
    got = c.attend(pages, q, batch.d_tables, batch.d_lengths)
    assert got[0, 1:3].isnan().all()
    keep = torch.ones(n, 4, dtype=torch.bool)
    keep[0, 1:3] = False
    assert torch.equal(got[keep.cuda()], clean[keep.cuda()])


# ------------------------------------------------------------------ the calls together

@pytest.mark.parametrize("bits,dtype,d", [(8, "bf16", 128), (4, "f16", 64), (8, "f32", 100)])
def test_a_prompt_and_its_answer_in_steps(bf, torch, bits, dtype, d):
    """Chunks of a prompt, then single tokens, each written and attended to: as if the sequence had been written at once."""
    heads, group, ps = 2, 3, 16
    steps = [[33, 5], [31, 64], [1, 1], [1, 0], [1, 1]]
    total = [sum(s[b] for s in steps) for b in (0, 1)]
    whole = Batch(torch, total, total, ps)
    rng = np.random.default_rng(0)
    k, v, q = (_rows(torch, rng, whole.T, h, d, dtype, "packed") for h in (heads, heads, heads * group))
    c = bf.PagedCache(bits, heads, d, ps)
    pages, at_once = c.new_pages(whole.count), c.new_pages(whole.count)
    c.write(at_once, k, v, whole.d_tables, whole.d_lengths, whole.d_indptr)
    want = c.attend(at_once, q, whole.d_tables, whole.d_lengths, whole.d_indptr)
    done = [0, 0]
    for news in steps:
        pick = torch.cat([torch.arange(int(whole.starts[b]) + done[b], int(whole.starts[b]) + done[b] + news[b]) for b in (0, 1)]).cuda()
        done = [done[b] + news[b] for b in (0, 1)]
        lengths = torch.tensor(done, dtype=torch.int64, device="cuda")
        indptr = torch.tensor([0, news[0], news[0] + news[1]], dtype=torch.int64, device="cuda")
        c.write(pages, k[pick], v[pick], whole.d_tables, lengths, indptr)
        got = c.attend(pages, q[pick], whole.d_tables, lengths, indptr)
        assert (got.float() - want[pick].float()).abs().max() <= 2 * (2 * WEIGHT[dtype] + HALF_ULP[dtype] + 2.0 ** -16) * v.float().abs().max()
    a, b = (c.read(p, whole.d_tables, whole.d_lengths, whole.T, whole.d_indptr) for p in (pages, at_once))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_pages_past_4_gib(bf, torch):
    heads, d, ps = 8, 128, 64
    c = bf.PagedCache(8, heads, d, ps)
    count = (5 << 30) // c.page_bytes
    pages = torch.zeros((count, c.page_bytes), dtype=torch.uint8, device="cuda")
    small = Batch(torch, [200], [200], ps)
    rng = np.random.default_rng(0)
    k, v, q = (_rows(torch, rng, 200, h, d, "bf16") for h in (heads, heads, heads))
    want = None
    for first in (0, count - small.count):
        tables = (torch.from_numpy(small.tables).cuda() + first).contiguous()
        c.write(pages, k, v, tables, small.d_lengths)
        got = (c.attend(pages, q, tables, small.d_lengths), c.attend(pages, q[-1:], tables, small.d_lengths),
               *c.read(pages, tables, small.d_lengths, 200))
        assert want is None or all(torch.equal(x, y) for x, y in zip(got, want))
        want = got
    # what lies between was left alone
    assert not pages[small.count:small.count + 3].any() and not pages[count - 2 * small.count:count - small.count].any()


def test_other_streams_and_replayed_graphs(bf, torch):
    batch = Batch(torch, [3000, 77, 500], [1, 1, 1], 16)
    heads, d = 2, 64
    c = bf.PagedCache(8, heads, d, 16)
    raw, _ = _filled(torch, batch, c, 8, heads, d, seed=1)
    rng = np.random.default_rng(2)
    k, v, q = (_rows(torch, rng, 3, h, d, "f16", "packed") for h in (heads, heads, 8))
    pages = torch.from_numpy(raw).cuda()
    c.write(pages, k, v, batch.d_tables, batch.d_lengths)
    want = c.attend(pages, q, batch.d_tables, batch.d_lengths)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = c.attend(pages, q, batch.d_tables, batch.d_lengths)
    side.synchronize()
    assert torch.equal(got, want)
    # a handle whose workspace is there, and one that has none and may not get one
    for handle, reserve in ((bf.PagedCache(8, heads, d, 16), True), (bf.PagedCache(8, heads, d, 16), False)):
        if reserve:
            handle.reserve()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        out = torch.zeros_like(q)
        back = [torch.zeros(3, heads, d, dtype=torch.float32, device="cuda") for _ in range(2)]
        with torch.cuda.graph(graph):
            handle.write(pages, k, v, batch.d_tables, batch.d_lengths)
            handle.attend(pages, q, batch.d_tables, batch.d_lengths, out=out)
            handle.read(pages, batch.d_tables, batch.d_lengths, 3, out=back)
        for i in range(4):
            k.copy_(torch.randn_like(k)), v.copy_(torch.randn_like(v)), q.copy_(torch.randn_like(q))
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            fresh = pages.clone()
            c.write(fresh, k, v, batch.d_tables, batch.d_lengths)
            assert torch.equal(fresh, pages)
            eager = c.attend(pages, q, batch.d_tables, batch.d_lengths)
            if reserve:
                assert torch.equal(out, eager), i
            else:   # without a workspace contexts are not split: other sums, the same within their rounding
                assert (out.float() - eager.float()).abs().max() <= 2.0 ** -8 * 4, i
            assert torch.equal(back[0], c.read(pages, batch.d_tables, batch.d_lengths, 3)[0])


def test_validate_refuses_a_broken_batch(bf, torch):
    batch = Batch(torch, [40, 20], [2, 3], 16)
    c = bf.PagedCache(8, 1, 64, 16)
    pages = c.new_pages(batch.count)
    k = torch.zeros(5, 1, 64, device="cuda")
    args = (batch.d_tables, batch.d_lengths, batch.d_indptr)
    assert c.check(pages, *args)
    c.set_option("validate", 1)
    c.write(pages, k, k, *args)
    c.attend(pages, k, *args)
    broken = []
    t = batch.d_tables.clone()
    t[0, 1] = batch.count
    broken.append((t, args[1], args[2]))
    t = batch.d_tables.clone()
    t[1, 0] = -1
    broken.append((t, args[1], args[2]))
    broken.append((args[0], torch.tensor([40, 16 * batch.width + 1], device="cuda"), args[2]))
    broken.append((args[0], torch.tensor([-1, 20], device="cuda"), args[2]))
    for p in ([0, 2, 4], [1, 2, 5], [0, 6, 5]):
        broken.append((args[0], args[1], torch.tensor(p, device="cuda")))
    for bad in broken:
        assert not c.check(pages, *bad, tokens=5)
        for call in (lambda: c.write(pages, k, k, *bad), lambda: c.attend(pages, k, *bad), lambda: c.read(pages, bad[0], bad[1], 5, bad[2])):
            with pytest.raises(bf.BifeatError) as e:
                call()
            assert e.value.status == bf.EINVAL
    # nothing was launched, and the handle still works
    assert c.attend(pages, k, *args).shape == k.shape


def test_no_tokens(bf, torch):
    c = bf.PagedCache(4, 2, 64, 16)
    pages = c.new_pages(1)
    none = torch.empty(0, 2, 64, device="cuda")
    tables, lengths = torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int64, device="cuda")
    c.write(pages, none, none, tables, lengths)
    assert c.attend(pages, none, tables, lengths).shape == (0, 2, 64)
    assert c.read(pages, tables, lengths, 0)[0].shape == (0, 2, 64)


def test_refusals_of_the_python_calls(bf, torch):
    c = bf.PagedCache(8, 2, 64, 16)
    pages = c.new_pages(4)
    tables, lengths = torch.zeros(2, 2, dtype=torch.int32, device="cuda"), torch.ones(2, dtype=torch.int64, device="cuda")
    x = torch.zeros(2, 2, 64, device="cuda")
    bad = [
        lambda: c.write(pages, x, x[:, :1], tables, lengths), lambda: c.write(pages, x, x.half(), tables, lengths),
        lambda: c.write(pages, x.double(), x.double(), tables, lengths), lambda: c.write(pages[:, 1:], x, x, tables, lengths),
        lambda: c.write(pages, x.transpose(1, 2).contiguous().transpose(1, 2), x, tables, lengths),
        lambda: c.write(pages, x.cpu(), x.cpu(), tables, lengths), lambda: c.write(pages, x, x, tables.long(), lengths),
        lambda: c.write(pages, x, x, tables, lengths.int()), lambda: c.write(pages, x, x, tables, lengths[:1]),
        lambda: c.write(pages, x, x, tables, lengths, torch.zeros(2, dtype=torch.int64, device="cuda")),
        lambda: c.attend(pages, x[:, :, :32], tables, lengths), lambda: c.attend(pages, x, tables, lengths, out=x.half()),
        lambda: c.attend(pages, x, tables, lengths, slopes=torch.zeros(3, device="cuda")),
        lambda: c.attend(pages, x, tables, lengths, prefix=torch.zeros(3, dtype=torch.int64, device="cuda")),
        lambda: c.attend(pages, x, tables[:, ::2], lengths), lambda: c.read(pages, tables, lengths, 2, out=(x, x[:1]))]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    for call in [lambda: c.write(pages, x[:1], x[:1], tables, lengths),             # 1 token, 2 sequences
                 lambda: c.attend(pages, x[:, :1], tables, lengths),               # 1 query head, 2 cached
                 lambda: c.attend(pages, x, tables, lengths, window=-1), lambda: c.attend(pages, x, tables, lengths, softcap=-1.0),
                 lambda: c.attend(pages, x, tables, lengths, scale=float("nan")), lambda: c.read(pages, tables, lengths, 3)]:
        with pytest.raises(bf.BifeatError) as e:
            call()
        assert e.value.status == bf.EINVAL


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("n", [1, 40])
def test_many_sequences(bf, torch, ragged, n):
    # more sequences and items than a workgroup has threads; in the ragged batch some bring nothing
    B, heads, d, ps = 700 if n == 1 else 300, 1, 32, 16
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(n, n + 90, B)]
    lengths[B // 2] = 900   # contexts are shared between workgroups
    news = [n] * B if not ragged else [int(x) for x in rng.integers(0, n + 1, B)]
    _attend_case(bf, torch, 8, heads, 2, d, ps, "f16", lengths, news, uniform=not ragged, seed=B)


@pytest.mark.parametrize("dtype,bits,d", [("f16", 4, 64), ("bf16", 8, 256), ("f32", 8, 128)])
@pytest.mark.parametrize("news", [[1, 1], [20, 20], [200, 90]])
@pytest.mark.parametrize("opts", [dict(window=300, prefix=[130, 700]), dict(window=64, slopes=True), dict(window=1000, prefix=[1, 0], cap=20.0)])
def test_attend_over_a_window_and_a_prefix_far_apart(bf, torch, news, opts, dtype, bits, d):
    _attend_case(bf, torch, bits, 1, 2, d, 32, dtype, [2300, 1500], news, **opts)


def test_every_row_of_a_call_may_see_nothing(bf, torch):
    batch = Batch(torch, [0, 0], [3, 3], 16)
    c = bf.PagedCache(8, 1, 64, 16)
    pages = torch.full((batch.count, c.page_bytes), 255, dtype=torch.uint8, device="cuda")
    q = torch.randn(6, 2, 64, device="cuda")
    out = torch.full_like(q, 7.0)
    c.attend(pages, q, batch.d_tables, batch.d_lengths, out=out)
    assert not out.any()
    k = torch.randn(6, 1, 64, device="cuda")
    c.write(pages, k, k, batch.d_tables, batch.d_lengths)
    assert (pages == 255).all()
    assert not any(x.any() for x in c.read(pages, batch.d_tables, batch.d_lengths, 6))


def test_the_example(bf, torch):
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "cached_answers.py")
    spec = importlib.util.spec_from_file_location("cached_answers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    off = {bits: example.answer(bits, prompts=(70, 33, 5), tokens=6, chunk=32) for bits in (4, 8)}
    # logits against those without a cache: a value's level is 1 / 255 or 1 / 15 of its row's range, of which half is the most
    # that it is off by; two layers' worth, relative to the logits' size
    assert off[8] < 0.03 and off[8] < off[4] < 0.4
