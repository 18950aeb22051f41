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


@pytest.mark.parametrize("branches,n", [
    ([[0, 2, 1], [0]], 3), ([[0, 0], [0]], 3), ([[0, 3], [0]], 3), ([[-1, 0], [0]], 3), ([[0]], 3), ([[0], [0], [0]], 3), ([[0, 1, 2, 3], [0]], 3),
    ([[0], [0]], 0), ([[0], [0]], 60)])
def test_commit_refuses_what_is_no_branch(branches, n):
    """and leaves cache, positions and bounds as they were"""
    model = decoder()
    model.verify(torch.zeros(2, 3, dtype=torch.int32, device="cuda"), [[-1, 0, 1], [-1, 0, 0]])
    held, pos = list(model.held), model.seq_pos.clone()
    before = [t.clone() for t in model.cache._tensors]
    with pytest.raises(ValueError):
        model.commit(branches, n)
    assert model.held == held and torch.equal(model.seq_pos, pos) and all(torch.equal(a, b) for a, b in zip(before, model.cache._tensors))


def test_commit_takes_a_branch_and_none():
    model = decoder()
    model.verify(torch.zeros(2, 3, dtype=torch.int32, device="cuda"), [[-1, 0, 1], [-1, 0, 0]])
    model.commit([[0, 2], []], 3)
    assert model.held == [12, 7] and model.seq_pos.tolist() == [12, 7]
