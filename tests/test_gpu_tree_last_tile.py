"""Attention of drafted trees where the last tile of cache rows passes the end of the cache: rows that lie in the tile before too count
once, whatever they hold."""
import numpy as np
import pytest
import torch

from paper_2604_16498_amd import binding as F
from tree_inputs import ancestor_bits, cache_arrays, gpu, normal, parents, signed

pytestmark = pytest.mark.gpu


# rows of cache that tiles of 32 do not divide; `at`: the row that holds the odd element.  Rows 998 .. 1023 of 1030 are in two tiles, of
# which the second begins a share of its own where nine shares are dealt over the 18 units of two heads.
@pytest.mark.parametrize("store,value", [("bf16", float("inf")), ("bf16", float("-inf")), ("bf16", float("nan")),
                                         ("fp32", float("inf")), ("fp32", float("nan")), ("fp8", float("nan"))])
@pytest.mark.parametrize("B,n,Hq,Hkv,dh,pos,cap,at", [
    (1, 16, 2, 2, 128, 1014, 1030, 1017), (1, 16, 4, 2, 128, 1014, 1030, 1017), (1, 16, 2, 2, 64, 1014, 1030, 1020),
    (1, 16, 4, 2, 64, 1014, 1030, 1005), (1, 16, 2, 2, 128, 1014, 1030, 1000), (1, 12, 4, 2, 128, 1014, 1030, 999),
    (1, 7, 2, 2, 64, 90, 100, 93), (1, 7, 2, 2, 128, 90, 100, 70), (1, 13, 4, 2, 64, 90, 103, 101), (2, 1, 2, 2, 64, 32, 33, 5),
    (1, 5, 4, 2, 128, 640, 645, 641), (40, 3, 8, 8, 64, 34, 37, 35), (40, 3, 8, 8, 128, 34, 37, 20), (40, 20, 8, 8, 64, 60, 80, 63)])
def test_an_odd_element_counts_once(B, n, Hq, Hkv, dh, pos, cap, at, store, value):
    rng = np.random.default_rng(at)
    col, head = 3, 0
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    (k, v, ks, vs), _ = cache_arrays(rng, store, (B, Hkv, cap, dh))
    for bits in ([(2 << t) - 1 for t in range(n)], ancestor_bits(parents(rng, n))):
        held = v.clone()
        if store == "fp8":
            held.view(torch.uint8)[:, head, at, col] = 0x7f
        else:
            held[:, head, at, col] = value
        c = F.make_kv_cache(k, held, ks, vs)
        q = gpu(normal(rng, (B, n, Hq, dh), store != "fp32"), dt)
        out = torch.full((B, n, Hq * dh), 7.0, dtype=dt, device="cuda")
        ws = F.workspace(F.forge_attn_tree_workspace_bytes(c, Hq, n, pos))
        F.forge_attn_tree(c, q, out, torch.full((B,), pos, dtype=torch.int32, device="cuda"), pos,
                          visible=torch.tensor(signed([bits] * B), dtype=torch.int64, device="cuda"), workspace=ws)
        # fp64; the odd element counts as 0 in the sums, and those who see it get it
        rows, G = pos + n, Hq // Hkv
        kk, vv = ((t[:, :, :rows].float().double() * (1.0 if s is None else s[:, :, :rows, None].double())).cpu() for t, s in ((k, ks), (v, vs)))
        vv[:, head, at, col] = 0.0
        see = torch.ones(n, rows, dtype=torch.bool)
        for t in range(n):
            for j in range(n):
                see[t, pos + j] = bool(bits[t] >> j & 1)
        qq = q.double().cpu().view(B, n, Hkv, G, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, dh)
        p = torch.matmul(qq, kk.transpose(2, 3)).view(B, Hkv, G, n, rows) * dh ** -0.5
        p = p.masked_fill(~see, -torch.inf).softmax(-1).view(B, Hkv, G * n, rows)
        want, size = (torch.matmul(p, x).view(B, Hkv, G, n, dh).permute(0, 3, 1, 2, 4) for x in (vv, vv.abs()))
        want = want.contiguous()
        want[:, see[:, at], head, :, col] = value
        got = out.view(B, n, Hkv, G, dh).double().cpu()
        odd = ~torch.isfinite(want)
        assert odd.any() and (torch.isnan(got[odd]).all() if np.isnan(value) else torch.equal(got[odd], want[odd]))
        # 16-bit: weights and output are rounded to bf16, 2^-8 of sum P |v| each; scores and sums in fp32 add about 1e-5
        bound = 2e-5 * size + 1e-5 if store == "fp32" else (2 * 2.0 ** -8 * 1.02 + 2e-5) * size + 1e-6
        assert ((got - want).abs() <= bound)[~odd].all()
