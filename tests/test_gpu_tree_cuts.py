"""Attention of drafted trees in every kernel and every cut (tests/test_tree_plan.py shows that the calls take them), against fp64 on the
device; and where an infinity in a draft goes."""
import numpy as np
import pytest
import torch

from paper_2604_16498_amd import binding as F
from test_gpu_tree_shares import check_call, lengths
from tree_inputs import ancestor_bits, cache_arrays, gpu, normal, parents, signed
from tree_plan_cases import CASES, STORES

pytestmark = pytest.mark.gpu
ALL = [(store, case) for store, kind in STORES.items() for case, _ in CASES[kind]]


@pytest.mark.parametrize("store,case", ALL)
def test_every_cut(store, case):
    B, n, Hq, Hkv, dh, top = case
    rng = np.random.default_rng(top + n)
    for kind in ["ragged"] + (["one long"] if B > 5 and top > 512 else []):
        check_call(rng, store, B, n, Hq, Hkv, dh, lengths(rng, B, top, kind))


@pytest.mark.parametrize("store,case", [(s, c) for s, c in ALL if s != "int8" and c[1] > 1])
def test_an_infinity_in_every_cut(store, case):
    """One element of one draft's v in every second sequence, in the first and the last head; every other output keeps its bits."""
    B, n, Hq, Hkv, dh, top = case
    rng = np.random.default_rng(top + n + 1)
    pos, at, col = lengths(rng, B, top, "ragged"), n // 2, dh - 3
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    (k, v, ks, vs), _ = cache_arrays(rng, store, (B, Hkv, top + n + 3, dh))
    vis = [ancestor_bits(parents(rng, n)) for _ in range(B)]
    q = gpu(normal(rng, (B, n, Hq, dh), store != "fp32"), dt)
    c = F.make_kv_cache(k, v, ks, vs)
    ws = F.workspace(F.forge_attn_tree_workspace_bytes(c, Hq, n, top))
    bits, seq = torch.tensor(signed(vis), dtype=torch.int64, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda")
    outs, spoiled = [], range(B - 1, -1, -2)
    for spoil in (False, True):
        for b in spoiled:
            for h in {0, Hkv - 1}:
                if store == "fp8":
                    # (clean: a code of 0, as the element itself counts among the rest of its column; the type has no infinity)
                    v.view(torch.uint8)[b, h, pos[b] + at, col] = 0xff if spoil else 0
                else:
                    v[b, h, pos[b] + at, col] = float("-inf") if spoil else 0.0
        out = torch.empty(B, n, Hq * dh, dtype=dt, device="cuda")
        F.forge_attn_tree(c, q, out, seq, top, visible=bits, workspace=ws)
        outs.append(out.view(B, n, Hkv, Hq // Hkv, dh))
    hit = torch.zeros_like(outs[0], dtype=torch.bool)
    for b in spoiled:
        for t in range(n):
            for h in (0, Hkv - 1):
                hit[b, t, h, :, col] = bool(vis[b][t] >> at & 1)
    assert hit.any() and torch.equal(outs[0][~hit], outs[1][~hit]) and torch.isfinite(outs[0]).all()
    assert (torch.isnan(outs[1][hit]) if store == "fp8" else outs[1][hit] == float("-inf")).all()
