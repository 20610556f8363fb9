"""The example that runs products, turned keys, attention, routing and experts together is as near the same weights in full precision as a cache of
few bits lets it be, and a step that is put together wrongly is not."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PROMPTS, TOKENS = (70, 33, 5), 6


@pytest.fixture()
def example(monkeypatch):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_answers.py")
    spec = importlib.util.spec_from_file_location("packed_answers", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)

    class Decided(module.Model):
        """Biases that leave no doubt about the experts (scores are within 1), in each layer others: the two precisions choose alike."""

        def __init__(self, device, seed=0):
            super().__init__(device, seed)
            for p, best in zip(self.layers, ((5, 2), (0, 7))):
                p["bias"] = 0 * p["bias"]
                p["bias"][list(best)] = 4.0

    monkeypatch.setattr(module, "Model", Decided)
    return module


def _limits(bits):
    """Keys and values in `bits` bits are off by a step / sqrt(12) of a row's range, which is 4.8 deviations for 64 normal columns; rows have deviation 1.
    Scores q k / 8 are then off by that too, so that the attention's result is off by sqrt(2) of it relative to its own size, which for n positions of
    scores of deviation 1 is sqrt(sum of squared weights), sqrt(e / n), beside x of size 1.  Two layers; the experts pass an error of x on once.  Fp16 roundings
    are 2^-12 each, a dozen of them."""
    off = 4.8 / (2 ** bits - 1) / 12 ** 0.5
    return [2 * 2 * 2 ** 0.5 * off * (2.72 / (n + TOKENS)) ** 0.5 + 12 ** 0.5 * 2.0 ** -12 for n in PROMPTS]


@pytest.mark.parametrize("bits", [8, 4])
def test_logits_are_near_full_precision(example, bits):
    off = example.answer(bits, prompts=PROMPTS, tokens=TOKENS, chunk=32)
    assert all(a <= b for a, b in zip(off, _limits(bits))), (off, _limits(bits))


@pytest.mark.parametrize("wrong", ["pairs", "frequencies", "experts", "weights"])
def test_a_wrong_step_is_not_near(example, wrong, monkeypatch):
    bf = example.bf
    append, route = bf.PagedCache.append, bf.route
    if wrong == "pairs":
        monkeypatch.setattr(bf.PagedCache, "append", lambda self, *args: append(self, *args, interleaved=True))
    elif wrong == "frequencies":
        monkeypatch.setattr(bf.PagedCache, "append", lambda self, pages, q, k, v, f, *rest: append(self, pages, q, k, v, 1.5 * f, *rest))
    elif wrong == "experts":
        monkeypatch.setattr(bf, "route", lambda *args, **kw: ((r := route(*args, **kw))[0].sub(1).remainder(example.EXPERTS), r[1]))
    else:
        monkeypatch.setattr(bf, "route", lambda *args, **kw: ((r := route(*args, **kw))[0], r[1] * 1.25))
    off = example.answer(8, prompts=PROMPTS, tokens=TOKENS, chunk=32)
    assert all(a > 2 * b for a, b in zip(off, _limits(8))), (off, _limits(8))
