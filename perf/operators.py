"""What is measured of the paged cache of keys and values in few bits: the calls that a program which
generates text makes of it, at the sizes that it meets, from one token to whole prompts.

A case is a dict of plain values; `kind` says which call it makes:

  append   the keys and values of new tokens quantised into their pages, and read back as the values
           that they now stand for
  read     keys and values of whole contexts read back
  attend   attention of new tokens over the cache, their own keys and values in it already

Cached sequences: `B` of them, up to `ctx` tokens long (`ragged`: lengths spread between an eighth of
that and all of it), of which the last `n` are new (`ragged`: a batch of prompts and of single tokens,
as a server mixes them). A page holds `page` tokens of all heads; a sequence's pages lie anywhere. What
no token was written to yet holds arbitrary bytes.

A page is, head after head: codes of the keys [page][row], codes of the values [page][row], then 32-bit
floats key scale [page], key minimum [page], value scale [page], value minimum [page]; a row is
head_dim codes of `bits` bits, the first column in the lowest bits, filled up to 16 bytes with zeros.
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _case(name, kind, B, n, ctx, heads, d, **kw):
    case = {"name": name, "kind": kind, "B": B, "n": n, "ctx": ctx, "heads": heads, "group": 1, "d": d, "bits": 8,
            "page": 64, "dtype": "bf16", "ragged": False, "window": 0, "prefix": 0, "cap": 0.0, "slopes": False}
    case.update(kw)
    return case


def listed():
    return [
        # one token of one answer, 768 columns in 12 heads: a launch, and what the host needs for it
        _case("append_one_token", "append", 1, 1, 300, 12, 64, page=16, dtype="f16"),
        # a step of 256 answers at once, each at another length
        _case("append_256_answers", "append", 256, 1, 4096, 8, 128, bits=4, page=16, ragged=True),
        # prompts as they come in, some of one token
        _case("append_prompts", "append", 24, 2048, 2048, 8, 128, ragged=True),
        # one short context read back, to be attended to by code that takes whole tensors
        _case("read_one_context", "read", 1, 777, 777, 12, 64, bits=4, page=16, dtype="f32"),
        # the contexts of a batch read back
        _case("read_32_contexts", "read", 32, 8192, 8192, 8, 128, ragged=True),
        # one token of one answer, early in it
        _case("attend_one_token", "attend", 1, 1, 300, 12, 64, page=16, dtype="f16"),
        # a step of 64 answers, four query heads a cached one
        _case("attend_64_answers", "attend", 64, 1, 8192, 8, 128, group=4, ragged=True),
        # a step of four answers over very long contexts in 4 bits
        _case("attend_long_contexts", "attend", 4, 1, 131072, 8, 128, group=8, bits=4, page=128),
        # five drafted tokens of 32 answers checked at once, a sliding window and a prefix, capped scores
        _case("attend_drafts_window", "attend", 32, 5, 8192, 4, 256, group=4, bits=4, page=32, dtype="f16", ragged=True,
              window=1024, prefix=128, cap=30.0),
        # a chunk of a long prompt over what came before it
        _case("attend_chunk", "attend", 1, 2048, 32768, 8, 128, group=4),
        # a mixed batch: prompts of up to 2048 tokens beside single tokens, a bias by distance
        _case("attend_mixed_batch", "attend", 16, 2048, 4096, 12, 64, dtype="f16", ragged=True, slopes=True),
        # odd sizes in 32 bits: 100 columns, 77 new tokens
        _case("attend_odd_32bit", "attend", 3, 77, 1001, 2, 100, group=5, bits=4, page=16, dtype="f32", prefix=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "read", "attend", "attend", "attend"])
    group = rng.choice([1, 2, 4, 4, 5, 8]) if kind == "attend" else 1
    ctx = _log_uniform(rng, 16, 131072 if kind == "attend" else 8192)
    B = _log_uniform(rng, 1, 256)
    n = ctx if kind == "read" else rng.choice([1, 1, rng.randint(2, 8), _log_uniform(rng, 9, 2048)])
    case = _case("", kind, B, min(n, ctx), ctx, rng.choice([1, 2, 4, 8, 8, 12]),
                 rng.choice([64, 64, 80, 100, 128, 128, 128, 256, rng.randint(17, 255)]), group=group,
                 bits=rng.choice([4, 8]), page=rng.choice([16, 32, 64, 128]), dtype=rng.choice(["f32", "f16", "f16", "bf16", "bf16"]),
                 ragged=rng.random() < 0.6)
    del case["name"]
    if kind == "attend":
        case["window"] = rng.choice([0, 0, _log_uniform(rng, 64, 4096)])
        case["prefix"] = rng.choice([0, 0, rng.randint(1, 300)])
        case["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        case["slopes"] = rng.random() < 0.3
    # no dearer than the listed ones of the same kind: in bytes, in operations, and in what the plain form unfolds
    same = [c for c in listed() if c["kind"] == kind]
    most = [max(f(c) for c in same) for f in (lambda c: work(c)["bytes"], lambda c: work(c)["flops"], _unfolded)]
    while work(case)["bytes"] > most[0] or work(case)["flops"] > most[1] or _unfolded(case) > most[2]:
        if case["B"] > 1:
            case["B"] = case["B"] // 2
        elif case["n"] > 1 and kind != "read":
            case["n"] = case["n"] // 2
        else:
            case["ctx"] = max(1, case["ctx"] // 2)
            case["n"] = min(case["n"], case["ctx"])
    return case


def _unfolded(c):
    """Scores, and decoded keys, of a whole batch as one tensor."""
    return c["B"] * c["heads"] * c["ctx"] * max(c["group"] * (c["n"] if c["kind"] == "attend" else 0), c["d"])


@functools.lru_cache(maxsize=256)
def _sizes(B, n, ctx, ragged, kind):
    """Lengths of the sequences with their new tokens, and how many are new, the same for every seed."""
    r = random.Random(1000003 * B + 1009 * ctx + n)
    lengths = [r.randint(max(1, ctx // 8), ctx) if ragged else ctx for _ in range(B)]
    lengths[r.randrange(B)] = ctx
    if kind == "read":
        news = list(lengths)
    elif ragged and n > 8:
        news = [min(m, 1 if r.random() < 0.5 else r.randint(1, n)) for m in lengths]
        longest = max(range(B), key=lambda b: lengths[b])
        news[longest] = min(n, lengths[longest])
    else:
        news = [min(n, m) for m in lengths]
    return lengths, news


def _of(case):
    lengths, news = _sizes(case["B"], case["n"], case["ctx"], case["ragged"], case["kind"])
    return lengths, news


def _row_bytes(case):
    return (case["d"] * case["bits"] + 127) // 128 * 16


def work(case):
    lengths, news = _of(case)
    T, esz = sum(news), 4 if case["dtype"] == "f32" else 2
    cached = case["heads"] * (2 * _row_bytes(case) + 16)      # bytes of a token in the cache
    plain = 2 * case["heads"] * case["d"] * esz               # and of its keys and values as they come
    if case["kind"] == "append":
        return {"bytes": T * (2 * plain + 2 * cached), "flops": 8 * T * case["heads"] * case["d"]}
    if case["kind"] == "read":
        return {"bytes": T * (plain + cached), "flops": 4 * T * case["heads"] * case["d"]}
    w, pre = case["window"], case["prefix"]
    pairs = tokens = 0
    for m, n in zip(lengths, news):
        first = m - n
        seen = [min(p + 1, w) if w else p + 1 for p in range(first, m)]
        # of the prefix, what the window (or the order) leaves out is seen too
        pairs += sum(s + max(0, min(pre, m) - (p + 1)) + max(0, min(pre, p + 1 - s)) for s, p in zip(seen, range(first, m)))
        low = max(0, first + 1 - w) if w else 0
        tokens += m - max(0, low - min(pre, m))
    rows = T * case["heads"] * case["group"] * case["d"]
    return {"bytes": 2 * rows * esz + tokens * cached, "flops": 4 * pairs * case["heads"] * case["group"] * case["d"]}


# ------------------------------------------------------------------ inputs

def _pack(codes, row, bits):
    """[..., d] whole numbers -> [..., row] bytes."""
    codes = torch.nn.functional.pad(codes.to(torch.uint8), (0, row * 8 // bits - codes.shape[-1]))
    return codes if bits == 8 else codes[..., 0::2] | (codes[..., 1::2] << 4)


def _quantise(x, bits):
    """Codes, scale and minimum of each last-dimension vector, each step rounded to 32 bits."""
    x = x.float()
    top = float((1 << bits) - 1)
    low = x.amin(-1, keepdim=True)
    span = x.amax(-1, keepdim=True) - low
    tops = torch.full_like(span, top)
    inv = tops / span
    flat = ~torch.isfinite(inv)
    scale = torch.where(flat, torch.zeros_like(span), span / tops)
    inv = torch.where(flat, torch.zeros_like(span), inv)
    codes = torch.round((x - low) * inv).clamp(0.0, top)
    return codes, scale.squeeze(-1), low.squeeze(-1)


def _regions(pages, case):
    """Views of the pages: codes of keys and values [pages, heads, page, row], and the four floats [pages, heads, 4, page]."""
    ps, row, H = case["page"], _row_bytes(case), case["heads"]
    head = ps * (2 * row + 16)
    blocks = pages.view(pages.shape[0], H, head)
    codes = blocks[:, :, :2 * ps * row].unflatten(2, (2, ps, row))
    floats = pages.view(torch.float32).view(pages.shape[0], H, head // 4)[:, :, ps * row // 2:].unflatten(2, (4, ps))
    return codes[:, :, 0], codes[:, :, 1], floats


def _gen(seed, device):
    g = torch.Generator(device=device)
    g.manual_seed(int(seed))
    return g


def prepare(case, seed):
    dev = "cuda" if torch.cuda.is_available() else "cpu"
    g = _gen(seed, dev)
    H, G, d, ps, B = case["heads"], case["group"], case["d"], case["page"], case["B"]
    dt = DTYPES[case["dtype"]]
    lengths, news = _of(case)
    T, width = sum(news), -(-max(lengths) // ps)
    count = B * width + 3
    pages = torch.randint(0, 256, (count, H * ps * (2 * _row_bytes(case) + 16)), dtype=torch.uint8, device=dev, generator=g)
    tables = torch.randperm(count, device=dev, generator=g)[:B * width].view(B, width).to(torch.int32)
    s = {"case": case, "pages": pages, "tables": tables, "T": T, "nmax": max(news),
         "lengths": torch.tensor(lengths, dtype=torch.int64, device=dev)}
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    # batches whose sequences all bring as many tokens need no offsets
    s["indptr"] = torch.tensor(starts, dtype=torch.int64, device=dev) if len(set(news)) > 1 else None
    randn = lambda *shape: torch.randn(*shape, device=dev, generator=g)  # noqa: E731
    # a few columns of the keys are larger than the others and lie off zero; tokens' values differ in size
    column = 0.5 * torch.exp(0.6 * randn(H, d)) + 4.0 * (torch.rand(H, d, device=dev, generator=g) < 0.03)
    middle = 0.5 * randn(H, d) * column
    keys = lambda *lead: randn(*lead, H, d) * column + middle  # noqa: E731
    values = lambda *lead: randn(*lead, H, d) * torch.exp(0.5 * randn(*lead, H, 1))  # noqa: E731
    if case["kind"] != "append":
        k_codes, v_codes, floats = _regions(pages, case)
        ids = tables.long().view(-1)
        step = max(1, (1 << 27) // (ps * H * d))
        for at in range(0, ids.numel(), step):
            part = ids[at:at + step]
            for which, (region, made) in enumerate(((k_codes, keys), (v_codes, values))):
                codes, scale, low = _quantise(made(part.numel(), ps).to(dt), case["bits"])
                region[part] = _pack(codes, _row_bytes(case), case["bits"]).transpose(1, 2)
                floats[part, :, 2 * which] = scale.transpose(1, 2)
                floats[part, :, 2 * which + 1] = low.transpose(1, 2)
        # the room behind a sequence's last token was never written
        for b, m in enumerate(lengths):
            slots = torch.arange(m, width * ps, device=dev)
            page, slot = tables[b].long()[slots // ps], slots % ps
            for region in (k_codes, v_codes):
                region[page, :, slot] = torch.randint(0, 256, (slots.numel(), H, region.shape[-1]), dtype=torch.uint8, device=dev, generator=g)
            floats[page, :, :, slot] = float("nan")
    if case["kind"] == "read":
        return s
    # queries, keys and values come out of one projection, side by side
    joined = torch.empty(T, H * (G + 2), d, dtype=dt, device=dev)
    s["q"], s["k"], s["v"] = joined[:, :H * G], joined[:, H * G:H * (G + 1)], joined[:, H * (G + 1):]
    s["q"].copy_(randn(T, H * G, d) / column.repeat_interleave(G, 0).clamp(min=0.5) * 2.0)
    s["k"].copy_(keys(T))
    s["v"].copy_(values(T))
    s["prefix"] = s["slopes"] = None
    if case["prefix"]:
        s["prefix"] = torch.tensor([min(case["prefix"], m) for m in lengths], dtype=torch.int64, device=dev)
    if case["slopes"]:
        s["slopes"] = 2.0 ** (-8.0 * torch.arange(1, H * G + 1, dtype=torch.float32, device=dev) / (H * G))
    return s


# ------------------------------------------------------------------ the plain form

def _places(s):
    """Sequence, index among its new tokens, and position of every new token."""
    t = torch.arange(s["T"], device=s["pages"].device)
    if s["indptr"] is None:
        seq, first = t // s["nmax"], t // s["nmax"] * s["nmax"]
        n = torch.full_like(t, s["nmax"])
    else:
        seq = torch.searchsorted(s["indptr"], t, right=True) - 1
        first = s["indptr"][seq]
        n = s["indptr"][seq + 1] - first
    return seq, t - first, s["lengths"][seq] - n + t - first


def _values_of(codes, scale, low, bits, d):
    if bits == 4:
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    return low.unsqueeze(-1) + codes[..., :d].float() * scale.unsqueeze(-1)


def _read_plain(s):
    case = s["case"]
    k_codes, v_codes, floats = _regions(s["pages"], case)
    seq, _, pos = _places(s)
    page, slot = s["tables"][seq, pos // case["page"]].long(), pos % case["page"]
    f = floats[page, :, :, slot]
    out = (_values_of(k_codes[page, :, slot], f[:, :, 0], f[:, :, 1], case["bits"], case["d"]),
           _values_of(v_codes[page, :, slot], f[:, :, 2], f[:, :, 3], case["bits"], case["d"]))
    return tuple(x.to(DTYPES[case["dtype"]]) for x in out)


def _append_plain(s):
    case = s["case"]
    k_codes, v_codes, floats = _regions(s["pages"], case)
    seq, _, pos = _places(s)
    page, slot = s["tables"][seq, pos // case["page"]].long(), pos % case["page"]
    k, k_scale, k_low = _quantise(s["k"], case["bits"])
    v, v_scale, v_low = _quantise(s["v"], case["bits"])
    k_codes[page, :, slot] = _pack(k, _row_bytes(case), case["bits"])
    v_codes[page, :, slot] = _pack(v, _row_bytes(case), case["bits"])
    floats[page, :, :, slot] = torch.stack([k_scale, k_low, v_scale, v_low], -1)
    return _read_plain(s)


def _attend_plain(s):
    case = s["case"]
    H, G, d, B, ps = case["heads"], case["group"], case["d"], case["B"], case["page"]
    k_codes, v_codes, floats = _regions(s["pages"], case)
    ids = s["tables"].long()
    C = ids.shape[1] * ps
    j = torch.arange(C, device=ids.device)
    there = (j < s["lengths"][:, None])[:, None, :, None]                       # [B, 1, C, 1]
    f = floats[ids].permute(3, 0, 2, 1, 4).reshape(4, B, H, C)
    k = _values_of(k_codes[ids].transpose(1, 2).reshape(B, H, C, -1), f[0], f[1], case["bits"], d)
    k = torch.where(there, k, 0.0)
    v = _values_of(v_codes[ids].transpose(1, 2).reshape(B, H, C, -1), f[2], f[3], case["bits"], d)
    v = torch.where(there, v, 0.0)
    seq, i, pos = _places(s)
    q = torch.zeros(B, s["nmax"], H * G, d, device=ids.device)
    q[seq, i] = s["q"].float()
    at = torch.full((B, s["nmax"]), -1, dtype=torch.int64, device=ids.device)
    at[seq, i] = pos
    x = torch.matmul(q.view(B, -1, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, -1, d), k.transpose(2, 3)) * (1.0 / math.sqrt(d))
    x = x.view(B, H, G, -1, C)
    if case["cap"]:
        x = case["cap"] * torch.tanh(x / case["cap"])
    away = at[:, :, None] - j                                                    # [B, nmax, C]
    if s["slopes"] is not None:
        x = x - s["slopes"].view(1, H, G, 1, 1) * away[:, None, None].float()
    seen = away >= 0
    if case["window"]:
        seen = seen & (away < case["window"])
    if s["prefix"] is not None:
        seen = seen | (j < s["prefix"][:, None, None])
    seen = (seen & (j < s["lengths"][:, None, None]) & (at[:, :, None] >= 0))[:, None, None]
    x = x.masked_fill(~seen, float("-inf"))
    x = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-3e38))
    x = x / x.sum(-1, keepdim=True).clamp(min=1e-37)
    out = torch.matmul(x.view(B, H, -1, C), v).view(B, H, G, -1, d).permute(0, 3, 1, 2, 4).reshape(B, -1, H * G, d)
    return out[seq, i].to(DTYPES[case["dtype"]])


# ------------------------------------------------------------------ one pass

@functools.lru_cache(maxsize=64)
def _cache(bits, heads, d, page):
    """The handle that a program keeps for its cache."""
    import paper_2207_14696_amd as bf
    return bf.PagedCache(bits, heads, d, page)


def run(state):
    s, case = state, state["case"]
    if not own:
        return {"append": _append_plain, "read": _read_plain, "attend": _attend_plain}[case["kind"]](s)
    c = _cache(case["bits"], case["heads"], case["d"], case["page"])
    if case["kind"] == "attend":
        return c.attend(s["pages"], s["q"], s["tables"], s["lengths"], s["indptr"], softcap=case["cap"], window=case["window"],
                        prefix=s["prefix"], slopes=s["slopes"])
    if case["kind"] == "append":
        c.write(s["pages"], s["k"], s["v"], s["tables"], s["lengths"], s["indptr"])
    return c.read(s["pages"], s["tables"], s["lengths"], s["T"], s["indptr"], dtype=DTYPES[case["dtype"]])


# ------------------------------------------------------------------ the definition, in 64 bits

def _sequence(case, pages, table, which, first, last):
    """Cached keys (which = 0) or values (1) of positions [first, last) of one sequence, [tokens, heads, d] in 64 bits."""
    ps, H, d, bits = case["page"], case["heads"], case["d"], case["bits"]
    row = _row_bytes(case)
    raw = pages[table.long()].view(-1, H, ps * (2 * row + 16))
    codes = raw[:, :, which * ps * row:(which + 1) * ps * row].reshape(-1, H, ps, row).to(torch.int64)
    column = torch.arange(d, device=raw.device)
    codes = (codes[..., column * bits // 8] >> (column * bits % 8)) & ((1 << bits) - 1)
    tail = raw[:, :, 2 * ps * row:].contiguous().view(torch.float32).view(-1, H, 4, ps).double()
    got = tail[:, :, 2 * which + 1, :, None] + codes.double() * tail[:, :, 2 * which, :, None]
    return got.permute(0, 2, 1, 3).reshape(-1, H, d)[first:last]


def exact(case, seed):
    s = prepare(case, seed)
    lengths, news = _of(case)
    H, G, d = case["heads"], case["group"], case["d"]
    if case["kind"] == "append":
        got = []
        for x in (s["k"].double(), s["v"].double()):
            low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            top = 2 ** case["bits"] - 1
            step = (high - low) / top
            got.append(low + step * torch.round((x - low) / step).nan_to_num(0.0))
        return tuple(got)
    if case["kind"] == "read":
        return tuple(torch.cat([_sequence(case, s["pages"], s["tables"][b], w, m - n, m) for b, (m, n) in enumerate(zip(lengths, news))])
                     for w in (0, 1))
    rows, start = [], 0
    for b, (m, n) in enumerate(zip(lengths, news)):
        k, v = (_sequence(case, s["pages"], s["tables"][b], w, 0, m) for w in (0, 1))
        q = s["q"][start:start + n].double()
        start += n
        pos = torch.arange(m - n, m, device=q.device)[:, None]
        key = torch.arange(m, device=q.device)[None, :]
        seen = key <= pos
        if case["window"]:
            seen &= key > pos - case["window"]
        if case["prefix"]:
            seen |= key < case["prefix"]
        out = torch.zeros(n, H * G, d, dtype=torch.float64, device=q.device)
        for h in range(H * G):
            x = q[:, h] @ k[:, h // G].T / math.sqrt(d)
            if case["cap"]:
                x = torch.tanh(x / case["cap"]) * case["cap"]
            if case["slopes"]:
                x = x + 2.0 ** (-8.0 * (h + 1) / (H * G)) * (key - pos)
            out[:, h] = torch.softmax(torch.where(seen, x, -math.inf), -1) @ v[:, h // G]
        rows.append(out)
    return torch.cat(rows)
