"""Generation with drafted trees against one token a pass, where the two may differ: other kernels add up in another order and an
int8 code may flip, so a token may only differ where the logits of both are a rounding apart."""
import numpy as np
import pytest
import torch

from paper_2604_16498_amd import inputs as I
from paper_2604_16498_amd import tree_decode as T

pytestmark = pytest.mark.gpu

SHAPE = I.BlockShape(256, 4, 2, 64, 512, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=10000.0, has_bias=False)
LAYERS = 3


class Keeping(T.TreeDecoder):
    def _choose(self, h):
        self.rows = h.clone()
        return super()._choose(h)


def logits_after(weights, top, store, tokens):
    """fp64 head over the last row that a prompt of these tokens gives"""
    model = Keeping(SHAPE, weights, top, 1, 512, store=store)
    model.prompt(torch.tensor([tokens], dtype=torch.int32, device="cuda"), [len(tokens)])
    x = model.rows[0, -1].double()
    y = x * (x.pow(2).mean() + SHAPE.eps).rsqrt() * top["normf_g"].double()
    return top["wte"].double() @ y


@pytest.mark.parametrize("store", ["int8", "fp8", "same"])
@pytest.mark.parametrize("seed,vocab", [(1, 97), (2, 1000), (3, 5000)])
def test_tokens_differ_only_where_logits_tie(seed, vocab, store):
    weights, top = T.random_model(SHAPE, LAYERS, vocab, seed=seed)
    B, S, lengths = 3, 80, [80, 33, 5]
    ids = torch.randint(0, vocab, (B, S), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()
    make = lambda: T.TreeDecoder(SHAPE, weights, top, B, 512, store=store)
    model = make()
    plain = T.generate(model, model.prompt(ids, lengths), 30, lambda tokens: ([], []))

    def draft(tokens):
        here = [p for p in plain if p[:len(tokens)] == tokens]
        right = here[0][len(tokens):len(tokens) + 4] if here else []
        wrong = [(t + 1) % vocab for t in right]
        return wrong + right, [max(0, i) for i in range(len(wrong))] + [0 if i == 0 else len(wrong) + i for i in range(len(right))]
    model = make()
    trees = T.generate(model, model.prompt(ids, lengths), 8, draft)
    agreed = 0
    for b, (one, other) in enumerate(zip(plain, trees)):
        m = min(len(one), len(other))
        first = next((i for i in range(m) if one[i] != other[i]), m)
        agreed += first
        if first == m:
            continue
        prefix = ids[b, :lengths[b]].tolist() + one[:first]
        logits = logits_after(weights, top, store, prefix)
        # the parity bound of a layer, 2e-2 of a value or of the rms, for every layer and the head, in both runs; the codes of an 8-bit
        # cache, half a step of 1/127 (int8) or 1/16 (fp8) of it, come on top
        step = {"same": 0.0, "int8": 0.5 / 127, "fp8": 0.5 / 16}[store]
        rms = float(logits.pow(2).mean().sqrt())
        slack = sum(2 * (2e-2 + step) * (LAYERS + 1) * max(abs(float(logits[t])), rms) for t in (one[first], other[first]))
        top_two = [float(logits[one[first]]), float(logits[other[first]])]
        assert abs(top_two[0] - top_two[1]) <= slack and max(top_two) >= float(logits.max()) - slack, (b, first, top_two, float(logits.max()))
    assert agreed >= B       # (the first token comes from the same prompt)
