"""Attention of drafted trees where one cached row outweighs all others by more than fp32 holds: an infinity in a draft reaches those that
see it, however the rows are cut into shares.  (Its weight is positive, if tiny; a share's weight may round to 0.)"""
import numpy as np
import pytest
import torch

from paper_2604_16498_amd import binding as F
from tree_inputs import ancestor_bits, gpu, normal, parents, signed
from tree_plan_cases import CASES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("at_end", [False, True])
@pytest.mark.parametrize("store,case", [(s, c) for s in ("bf16", "fp32") for c, (_, _, cut) in CASES[s] if cut != "each" and c[0] < 100])
def test_an_infinity_of_tiny_weight(store, case, at_end):
    B, n, Hq, Hkv, dh, top = case
    rng = np.random.default_rng(top)
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    cap, draft, col = top + n + 2, n // 2, 5
    k = torch.zeros(B, Hkv, cap, dh, dtype=dt, device="cuda")
    v = gpu(normal(rng, (B, Hkv, cap, dh), store != "fp32"), dt)
    loud = top - 1 if at_end else 0
    k[:, :, loud] = 40.0                                     # a score of 40 sqrt(dh) against 0: a weight of e^-320 or less for the rest
    v[:, 0, top + draft, col] = float("inf")
    vis = [ancestor_bits(parents(rng, n)) for _ in range(B)]
    c = F.make_kv_cache(k, v)
    q, out = torch.ones(B, n, Hq, dh, dtype=dt, device="cuda"), torch.empty(B, n, Hq * dh, dtype=dt, device="cuda")
    F.forge_attn_tree(c, q, out, torch.full((B,), top, dtype=torch.int32, device="cuda"), top,
                      visible=torch.tensor(signed(vis), dtype=torch.int64, device="cuda"),
                      workspace=F.workspace(F.forge_attn_tree_workspace_bytes(c, Hq, n, top)))
    want = v[:, None, :, loud].expand(B, n, Hkv, dh)[:, :, :, None].repeat(1, 1, 1, Hq // Hkv, 1)
    for b in range(B):
        for t in range(n):
            if vis[b][t] >> draft & 1:
                want[b, t, 0, :, col] = float("inf")
    same = out.view(want.shape) == want                     # one weight of 1: no rounding
    wrong = int((~same).sum())
    assert wrong == 0
