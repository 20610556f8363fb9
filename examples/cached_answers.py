"""Answers from a small language model whose keys and values are kept in 4 or 8 bits: prompts go in in chunks, of another
length each, then all sequences grow by a token a step.  Every step writes its keys and values into the pages and attends
to all that its sequence holds; the last logits are compared with a run without a cache, in full precision.

    python examples/cached_answers.py [bits]

The model is a stand-in: random weights, two layers, grouped query heads, a sliding window in the second layer."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2207_14696_amd as bf  # noqa: E402

LAYERS, WIDTH, HEADS, CACHED, DIM, WORDS, PAGE, WINDOW = 2, 256, 8, 2, 64, 512, 16, 48


class Model:
    def __init__(self, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *shape: torch.randn(*shape, device=device, generator=g) / shape[0] ** 0.5  # noqa: E731
        self.words = torch.randn(WORDS, WIDTH, device=device, generator=g)
        self.layers = [(w(WIDTH, (HEADS + 2 * CACHED) * DIM), w(HEADS * DIM, WIDTH), w(WIDTH, 4 * WIDTH), w(4 * WIDTH, WIDTH))
                       for _ in range(LAYERS)]

    def forward(self, ids, attend):
        """Logits of the tokens ids [T]; attend(layer, q, k, v) is given slices of the layer's joint projection."""
        x = self.words[ids]
        norm = lambda y: y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
        for i, (qkv, out, up, down) in enumerate(self.layers):
            joint = (norm(x) @ qkv).half().view(-1, HEADS + 2 * CACHED, DIM)
            y = attend(i, joint[:, :HEADS], joint[:, HEADS:HEADS + CACHED], joint[:, HEADS + CACHED:])
            x = x + y.float().reshape(-1, HEADS * DIM) @ out
            x = x + torch.relu(norm(x) @ up) @ down
        return norm(x) @ self.words.T


def window_of(layer):
    return WINDOW if layer else 0


class Sequences:
    """Cached sequences: a pool of pages a layer, which sequences take from as they grow."""

    def __init__(self, bits, count, most, device):
        self.cache = bf.PagedCache(bits, CACHED, DIM, PAGE)
        self.pages = [self.cache.new_pages(count * -(-most // PAGE), device) for _ in range(LAYERS)]
        self.free = list(range(self.pages[0].shape[0]))[::-1]
        self.lengths, self.held = [0] * count, [0] * count
        self.tables = torch.zeros(count, -(-most // PAGE), dtype=torch.int32, device=device)

    def step(self, model, tokens):
        """tokens: one list a sequence (empty ones among them).  The logits of all of them, one after another."""
        for b, new in enumerate(tokens):
            self.lengths[b] += len(new)
            while self.held[b] * PAGE < self.lengths[b]:
                self.tables[b, self.held[b]] = self.free.pop()
                self.held[b] += 1
        device = self.tables.device
        lengths = torch.tensor(self.lengths, device=device)
        indptr = torch.tensor([0] + [len(t) for t in tokens], device=device).cumsum(0)

        def attend(layer, q, k, v):
            self.cache.write(self.pages[layer], k, v, self.tables, lengths, indptr)
            return self.cache.attend(self.pages[layer], q, self.tables, lengths, indptr, window=window_of(layer))

        return model.forward(torch.tensor([t for new in tokens for t in new], device=device), attend)


def whole(model, ids):
    """The last logits of one sequence, all of it at once."""
    def attend(layer, q, k, v):
        q, k, v = (t.float().transpose(0, 1) for t in (q, k.repeat_interleave(HEADS // CACHED, 1), v.repeat_interleave(HEADS // CACHED, 1)))
        at = torch.arange(q.shape[1], device=q.device)
        away = at[:, None] - at
        seen = (away >= 0) & (away < (window_of(layer) or len(ids)))
        return torch.softmax((q @ k.transpose(1, 2) / DIM ** 0.5).masked_fill(~seen, -torch.inf), -1).matmul(v).transpose(0, 1).half()

    return model.forward(torch.tensor(ids, device=model.words.device), attend)[-1]


def answer(bits, prompts=(200, 37, 90, 1), tokens=16, chunk=64, device="cuda"):
    """How far the last logits are from those without a cache, relative to their size."""
    model = Model(device)
    g = torch.Generator().manual_seed(1)
    texts = [torch.randint(0, WORDS, (n,), generator=g).tolist() for n in prompts]
    s = Sequences(bits, len(texts), max(prompts) + tokens, device)
    done = [0] * len(texts)
    last = [None] * len(texts)
    for _ in range(-(-max(prompts) // chunk) + tokens):
        new = []
        for b, text in enumerate(texts):
            if done[b] == len(text) and len(text) < prompts[b] + tokens:
                text.append(int(last[b].argmax()))      # the prompt is in: an answer, token by token
            new.append(text[done[b]:done[b] + chunk])
            done[b] += len(new[-1])
        if not any(new):
            break
        logits = s.step(model, new)
        at = 0
        for b, part in enumerate(new):
            at += len(part)
            if part:
                last[b] = logits[at - 1]
    off = [float((last[b] - (want := whole(model, text))).norm() / want.norm()) for b, text in enumerate(texts)]
    return max(off)


if __name__ == "__main__":
    for bits in [int(sys.argv[1])] if len(sys.argv) > 1 else [8, 4]:
        print(f"{bits} bits: logits within {answer(bits):.4f} of those without a cache")
