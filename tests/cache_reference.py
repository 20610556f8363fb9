"""The paged cache from its definition, in numpy and 64 bits (not collected by pytest)."""
from __future__ import annotations

import numpy as np


def quantise(x, bits):
    """Codes, scale and minimum of the last dimension's vectors, each step rounded to 32 bits once."""
    x = np.asarray(x, np.float32)
    top = np.float32((1 << bits) - 1)
    with np.errstate(all="ignore"):
        mn, mx = x.min(-1), x.max(-1)
        span = (mx - mn).astype(np.float32)
        inv, scale = (top / span).astype(np.float32), (span / top).astype(np.float32)
        flat = ~np.isfinite(inv)
        inv, scale = np.where(flat, np.float32(0), inv), np.where(flat, np.float32(0), scale)
        q = np.rint(((x - mn[..., None]).astype(np.float32) * inv[..., None]).astype(np.float32))
        q = np.clip(np.nan_to_num(q, nan=0.0), 0, top).astype(np.uint8)
        bad = ~np.isfinite(x).all(-1) | ~np.isfinite(span)
    q[bad] = 0
    return q, np.where(bad, np.float32(np.nan), scale), np.where(bad, np.float32(np.nan), mn)


def row_bytes(d, bits):
    return (d * bits + 127) // 128 * 16


def pack(codes, bits):
    d = codes.shape[-1]
    rb = row_bytes(d, bits)
    wide = np.zeros(codes.shape[:-1] + (rb * 8 // bits,), np.uint8)
    wide[..., :d] = codes
    return wide if bits == 8 else wide[..., 0::2] | wide[..., 1::2] << 4


class Pages:
    """The documented layout, one token at a time."""

    def __init__(self, raw, bits, heads, d, ps):
        self.raw, self.bits, self.heads, self.d, self.ps = raw, bits, heads, d, ps
        self.rb = row_bytes(d, bits)
        self.head_bytes = ps * (2 * self.rb + 16)

    def codes(self, page, head, which, slot):
        at = head * self.head_bytes + (which * self.ps + slot) * self.rb
        return self.raw[page, at:at + self.rb]

    def float_at(self, page, head, index, slot):
        at = head * self.head_bytes + 2 * self.ps * self.rb + 4 * (index * self.ps + slot)
        return self.raw[page, at:at + 4].view(np.float32)

    def put(self, page, slot, head, which, x):
        q, scale, mn = quantise(x, self.bits)
        self.codes(page, head, which, slot)[:] = pack(q, self.bits)
        self.float_at(page, head, 2 * which, slot)[:] = scale
        self.float_at(page, head, 2 * which + 1, slot)[:] = mn

    def get(self, page, slot, head, which):
        c = self.codes(page, head, which, slot).astype(np.int64)
        if self.bits == 4:
            c = np.stack([c & 15, c >> 4], -1).reshape(-1)
        s, mn = (float(self.float_at(page, head, 2 * which + i, slot)[0]) for i in (0, 1))
        return mn + c[:self.d].astype(np.float64) * s

    def sequence(self, table, length, which):
        """[length, heads, d] in 64 bits."""
        return np.stack([np.stack([self.get(table[j // self.ps], j % self.ps, h, which) for h in range(self.heads)])
                         for j in range(length)]) if length else np.zeros((0, self.heads, self.d))


def attend(q, keys, values, n, length, scale, softcap=0.0, window=0, prefix=0, slopes=None):
    """One sequence: q [n, query heads, d], keys and values [length, heads, d]; in 64 bits."""
    q = np.asarray(q, np.float64)
    Hq, G = q.shape[1], q.shape[1] // keys.shape[1]
    out = np.zeros((n, Hq, q.shape[2]))
    j = np.arange(length)
    for i in range(n):
        p = length - n + i
        if p < 0:
            continue
        seen = ((j <= p) & ((window == 0) | (j > p - window))) | (j < prefix)
        if not seen.any():
            continue
        at = j[seen]
        for h in range(Hq):
            x = scale * (keys[at, h // G] @ q[i, h])
            if softcap > 0:
                x = softcap * np.tanh(x / softcap)
            if slopes is not None:
                x = x + float(slopes[h]) * (at - p)
            w = np.exp(x - x.max())
            out[i, h] = (w / w.sum()) @ values[at, h // G]
    return out
