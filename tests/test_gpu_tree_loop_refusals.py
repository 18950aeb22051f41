"""What the loop over drafted trees refuses: trees and branches that do not belong to its batch would be answered wrongly."""
import pytest
import torch

from paper_2604_16498_amd import inputs as I
from paper_2604_16498_amd import tree_decode as T

pytestmark = pytest.mark.gpu

SHAPE = I.BlockShape(256, 4, 2, 64, 512, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=10000.0, has_bias=False)


def decoder(B=2, drafts=6):
    weights, top = T.random_model(SHAPE, 1, 50)
    model = T.TreeDecoder(SHAPE, weights, top, B, 64, drafts=drafts)
    model.prompt(torch.zeros(B, 10, dtype=torch.int32, device="cuda"), [10, 7][:B])
    return model


def test_verify_refuses_trees_of_another_batch():
    model = decoder()
    ids = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    good = [-1, 0, 1]
    model.verify(ids, [good, good])
    for bad in ([good], [good, good, good], []):
        with pytest.raises(ValueError):
            model.verify(ids, bad)
    with pytest.raises(ValueError):
        model.verify(ids[:1], [good])
