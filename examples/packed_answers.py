"""Answers from a small language model that is kept in few bits as a whole: projections and experts in 4, keys and values in 4 or 8.
A step of it is a product, keys turned to their positions on their way into the pages, attention over them, a product, and two
products of the experts that the router chooses, joined by its weights.  The last logits are compared with those of the same
weights in full precision.

    python examples/packed_answers.py [bits of the cache]

The model is a stand-in: random weights, two layers, grouped query heads, eight experts of which a token takes two."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2207_14696_amd as bf  # noqa: E402
from examples.cached_answers import Sequences  # noqa: E402

LAYERS, WIDTH, HEADS, CACHED, DIM, WORDS, PAGE, EXPERTS, TAKEN, HIDDEN = 2, 256, 8, 2, 64, 512, 16, 8, 2, 384


def norm(y):
    return y * torch.rsqrt(y.float().square().mean(-1, keepdim=True) + 1e-6)


class Model:
    """Packed weights, and what they stand for."""

    def __init__(self, device, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *shape: torch.randn(*shape, device=device, generator=g) / shape[-1] ** 0.5  # noqa: E731
        self.words = torch.randn(WORDS, WIDTH, device=device, generator=g)
        self.frequencies = (10000.0 ** (-torch.arange(DIM // 2, device=device, dtype=torch.float64) / (DIM // 2))).float()
        self.joint, self.out = bf.PackedLinear((HEADS + 2 * CACHED) * DIM, WIDTH, group=64), bf.PackedLinear(WIDTH, HEADS * DIM, group=64)
        self.up, self.down = bf.PackedLinear(HIDDEN, WIDTH, group=64, experts=EXPERTS), bf.PackedLinear(WIDTH, HIDDEN, group=64, experts=EXPERTS)
        self.layers = [{"joint": self.joint.pack(w(self.joint.out_features, WIDTH)), "out": self.out.pack(w(WIDTH, HEADS * DIM)),
                        "up": self.up.pack(w(EXPERTS, HIDDEN, WIDTH)), "down": self.down.pack(w(EXPERTS, WIDTH, HIDDEN)), "router": w(WIDTH, EXPERTS),
                        "bias": 0.02 * torch.randn(EXPERTS, device=device, generator=g)} for _ in range(LAYERS)]

    def forward(self, ids, attend):
        """Logits of the tokens ids [T]; attend(layer, q, k, v) is given slices of the layer's joint projection."""
        x = self.words[ids]
        for i, p in enumerate(self.layers):
            rows = self.joint.multiply(p["joint"], norm(x).half()).view(-1, HEADS + 2 * CACHED, DIM)
            y = attend(i, rows[:, :HEADS], rows[:, HEADS:HEADS + CACHED], rows[:, HEADS + CACHED:])
            x = x + self.out.multiply(p["out"], y.reshape(-1, HEADS * DIM))
            z = norm(x)
            chosen, weights = bf.route(z @ p["router"], TAKEN, score="sigmoid", bias=p["bias"])
            hidden = torch.relu(self.up.multiply_experts(p["up"], z.half(), chosen))
            x = x + self.down.multiply_experts(p["down"], hidden, chosen, weights)
        return norm(x) @ self.words.T

    def whole(self, ids):
        """The last logits of one sequence, all of it at once, of the same weights in 32 bits and without a cache."""
        x = self.words[torch.tensor(ids, device=self.words.device)]
        T = len(ids)
        angle = torch.outer(torch.arange(T, device=x.device).double(), self.frequencies.double())
        cos, sin = (f(angle).float()[:, None] for f in (torch.cos, torch.sin))
        turn = lambda t: torch.cat([t[..., :DIM // 2] * cos - t[..., DIM // 2:] * sin, t[..., :DIM // 2] * sin + t[..., DIM // 2:] * cos], -1)  # noqa: E731
        seen = torch.ones(T, T, dtype=torch.bool, device=x.device).tril()
        for p in self.layers:
            rows = (norm(x) @ self.joint.unpack(p["joint"]).T).view(T, -1, DIM)
            q, k, v = turn(rows[:, :HEADS]), turn(rows[:, HEADS:HEADS + CACHED]), rows[:, HEADS + CACHED:]
            q, k, v = (t.transpose(0, 1).contiguous() for t in (q, k.repeat_interleave(HEADS // CACHED, 1), v.repeat_interleave(HEADS // CACHED, 1)))
            y = torch.softmax((q @ k.transpose(1, 2).contiguous() / DIM ** 0.5).masked_fill(~seen, -torch.inf), -1) @ v
            x = x + y.transpose(0, 1).reshape(T, -1) @ self.out.unpack(p["out"]).T
            z = norm(x)
            score = torch.sigmoid(z @ p["router"])
            chosen = (score + p["bias"]).topk(TAKEN).indices
            weights = torch.zeros_like(score).scatter(1, chosen, score.gather(1, chosen) / score.gather(1, chosen).sum(-1, keepdim=True))
            up, down = self.up.unpack(p["up"]), self.down.unpack(p["down"])
            x = x + sum(weights[:, e, None] * (torch.relu(z @ up[e].T) @ down[e].T) for e in range(EXPERTS))
        return (norm(x) @ self.words.T)[-1]


class Answers(Sequences):
    """The sequences of ``cached_answers.py``, their keys turned on their way into the cache."""

    def step(self, model, tokens):
        lengths, indptr, ids = self.grow(tokens)

        def attend(layer, q, k, v):
            q = self.cache.append(self.pages[layer], q, k, v, model.frequencies, self.tables, lengths, indptr)
            return self.cache.attend(self.pages[layer], q, self.tables, lengths, indptr)

        return model.forward(ids, attend)


def answer(bits, prompts=(200, 37, 90, 1), tokens=16, chunk=64, device="cuda"):
    """How far the last logits are from those in full precision, relative to their size, for each sequence."""
    model = Model(device)
    g = torch.Generator().manual_seed(1)
    texts = [torch.randint(0, WORDS, (n,), generator=g).tolist() for n in prompts]
    s = Answers(bits, len(texts), max(prompts) + tokens, device)
    done, last = [0] * len(texts), [None] * len(texts)
    for _ in range(-(-max(prompts) // chunk) + tokens):
        new = []
        for b, text in enumerate(texts):
            if done[b] == len(text) and len(text) < prompts[b] + tokens:
                text.append(int(last[b].argmax()))      # the prompt is in: an answer, token by token
            new.append(text[done[b]:done[b] + chunk])
            done[b] += len(new[-1])
        if not any(new):
            break
        logits, at = s.step(model, new), 0
        for b, part in enumerate(new):
            at += len(part)
            if part:
                last[b] = logits[at - 1]
    return [float((last[b] - (want := model.whole(text))).norm() / want.norm()) for b, text in enumerate(texts)]


if __name__ == "__main__":
    for bits in [int(sys.argv[1])] if len(sys.argv) > 1 else [8, 4]:
        print(f"cache of {bits} bits: logits within {', '.join(f'{off:.4f}' for off in answer(bits))} of those in full precision")
