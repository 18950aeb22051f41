"""Attention of drafted trees where its work is cut in other ways: many sequences, one long among short ones, whole pairs and shares, blocks of
every size, caches without a row to spare.  Against fp64 on the device; all rows that no token sees hold NaN."""
import numpy as np
import pytest
import torch

from paper_2604_16498_amd import binding as F
from tree_inputs import ancestor_bits, cache_arrays, gpu, normal, parents, signed

pytestmark = pytest.mark.gpu

STORES = ["int8", "fp8", "bf16", "fp32"]


def lengths(rng, B, top, kind):
    if kind == "one long":
        pos = rng.integers(0, 50, B)
        pos[B // 3] = top
    elif kind == "alike":
        pos = np.full(B, top)
    else:
        pos = rng.integers(0, top + 1, B)
        pos[rng.integers(0, B)] = top
    return [int(p) for p in pos]


def check_call(rng, store, B, n, Hq, Hkv, dh, pos, max_pos=None, spare=3):
    max_pos = max(pos) if max_pos is None else max_pos
    cap = max_pos + n + spare
    (k, v, ks, vs), _ = cache_arrays(rng, store, (B, Hkv, cap, dh))
    seen = torch.arange(cap, device="cuda")[None] < torch.tensor(pos, device="cuda")[:, None] + n
    dead = ~seen[:, None, :].expand(B, Hkv, cap)
    for t in (ks, vs) if store in ("int8", "fp8") else (k, v):
        t[dead] = float("nan")
    if store == "fp8":
        for t in (k, v):
            t.view(torch.uint8)[dead] = 0x7f
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    q = gpu(normal(rng, (B, n, Hq, dh), store != "fp32"), dt)
    vis = [ancestor_bits(parents(rng, n)) for _ in range(B)]
    c = F.make_kv_cache(k, v, ks, vs)
    ws = F.workspace(F.forge_attn_tree_workspace_bytes(c, Hq, n, max_pos))
    if ws is not None:
        ws.fill_(255)                                             # NaN wherever it is read before it is written
    out = torch.full((B, n, Hq * dh), 7.0, dtype=dt, device="cuda")
    bits = torch.tensor(signed(vis), dtype=torch.int64, device="cuda")
    F.forge_attn_tree(c, q, out, torch.tensor(pos, dtype=torch.int32, device="cuda"), max_pos, visible=bits, workspace=ws)
    G = Hq // Hkv
    for b, p in enumerate(pos):
        rows = p + n
        kk, vv = ((t[b, :, :rows].float().double() * (1.0 if s is None else s[b, :, :rows, None].double())) for t, s in ((k, ks), (v, vs)))
        qq = q[b].double().view(n, Hkv, G, dh).permute(1, 2, 0, 3).reshape(Hkv, G * n, dh)
        s = torch.matmul(qq, kk.transpose(1, 2).contiguous()) * dh ** -0.5
        draft = torch.arange(rows, device="cuda") - p
        ok = (draft[None] < 0) | ((bits[b][:, None] >> draft.clamp(min=0)[None]) & 1).bool()
        s = s.view(Hkv, G, n, rows).masked_fill(~ok, -torch.inf).softmax(-1).view(Hkv, G * n, rows)
        want, size = (torch.matmul(s, x).view(Hkv, G, n, dh).permute(2, 0, 1, 3).reshape(n, Hq * dh) for x in (vv, vv.abs()))
        err = (out[b].double() - want).abs()
        # 16-bit: weights and output are rounded to bf16, 2^-8 of sum P |v| each; scores and sums in fp32 add about 1e-5
        bound = 2e-5 * size + 1e-5 if store == "fp32" else (2 * 2.0 ** -8 * 1.02 + 2e-5) * size + 1e-6
        assert (err <= bound).all(), (b, p, float((err - bound).max()))        # (false for NaN)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("B,n,Hq,Hkv,dh,top,kind", [
    (300, 3, 4, 2, 64, 700, "ragged"), (256, 1, 2, 1, 128, 900, "ragged"), (257, 2, 2, 1, 64, 600, "ragged"), (65, 1, 8, 8, 64, 800, "ragged"),
    (64, 1, 8, 8, 128, 1000, "ragged"), (48, 8, 16, 8, 128, 700, "ragged"), (40, 1, 4, 1, 128, 6000, "one long"), (40, 12, 8, 2, 64, 6000, "one long"),
    (9, 20, 8, 1, 128, 4000, "one long"), (7, 5, 3, 3, 128, 2500, "alike"), (70, 9, 4, 1, 128, 1100, "ragged"), (100, 40, 4, 1, 64, 600, "ragged")])
def test_cut_over_sequences(B, n, Hq, Hkv, dh, top, kind, store):
    rng = np.random.default_rng(B + n)
    check_call(rng, store, B, n, Hq, Hkv, dh, lengths(rng, B, top, kind))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("B,n,Hq,Hkv,dh,top", [
    (1, 64, 8, 1, 128, 3000), (3, 33, 8, 1, 64, 5000), (20, 64, 6, 1, 128, 513), (2, 64, 5, 1, 128, 1025), (5, 26, 12, 2, 64, 1500),
    (130, 40, 4, 1, 128, 520), (33, 50, 16, 2, 64, 640), (1, 63, 17, 1, 128, 2049)])
def test_many_query_rows(B, n, Hq, Hkv, dh, top, store):
    rng = np.random.default_rng(B + n + 1)
    check_call(rng, store, B, n, Hq, Hkv, dh, lengths(rng, B, top, "ragged"))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("B,n,Hq,Hkv,dh,pos", [
    (1, 1, 1, 1, 64, [0]), (2, 1, 8, 2, 128, [3, 0]), (2, 5, 4, 1, 64, [10, 26]), (1, 31, 4, 2, 128, [0]), (1, 16, 3, 1, 128, [16]), (2, 64, 2, 1, 64, [0, 63]),
    (3, 7, 4, 4, 128, [600, 0, 999]), (4, 24, 4, 1, 128, [1000, 31, 32, 33])])
def test_no_row_to_spare(B, n, Hq, Hkv, dh, pos, store):
    """cap is the last row of the longest sequence, also below one tile"""
    check_call(np.random.default_rng(n), store, B, n, Hq, Hkv, dh, pos, spare=0)


@pytest.mark.parametrize("store", ["int8", "bf16"])
def test_a_workspace_serves_shorter_lengths(store):
    """positions far below max_pos: the cut is made for longer ones, and there are fewer rows than shares"""
    for n in (1, 40):
        for pos in ([0, 5, 130], [0, 0, 0], [300, 2000, 1]):
            check_call(np.random.default_rng(n), store, 3, n, 8, 2, 128, pos, max_pos=6000)


@pytest.mark.parametrize("store", ["fp8", "bf16", "fp32"])
@pytest.mark.parametrize("n,Hq,pos", [(40, 8, [3000, 10]), (64, 6, [700, 130]), (12, 8, [5000, 3])])
def test_an_infinity_reaches_those_that_see_it(n, Hq, pos, store):
    """one element of one draft's v; every other output keeps its bits"""
    rng = np.random.default_rng(n)
    dh, Hkv, at, col = 128, 2, 7, 5
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    (k, v, ks, vs), _ = cache_arrays(rng, store, (2, Hkv, max(pos) + n, dh))
    vis = [ancestor_bits(parents(rng, n)) for _ in range(2)]
    q = gpu(normal(rng, (2, n, Hq, dh), store != "fp32"), dt)
    c = F.make_kv_cache(k, v, ks, vs)
    ws = F.workspace(F.forge_attn_tree_workspace_bytes(c, Hq, n, max(pos)))
    bits, seq = torch.tensor(signed(vis), dtype=torch.int64, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda")
    outs = []
    for spoil in (False, True):
        if spoil:
            for b, p in enumerate(pos):
                if store == "fp8":
                    v.view(torch.uint8)[b, 1, p + at, col] = 0xff        # NaN: the type has no infinity
                else:
                    v[b, 1, p + at, col] = float("-inf")
        out = torch.empty(2, n, Hq * dh, dtype=dt, device="cuda")
        F.forge_attn_tree(c, q, out, seq, max(pos), visible=bits, workspace=ws)
        outs.append(out.view(2, n, Hkv, Hq // Hkv, dh))
    hit = torch.zeros_like(outs[0], dtype=torch.bool)
    for b in range(2):
        for t in range(n):
            hit[b, t, 1, :, col] = bool(vis[b][t] >> at & 1)
    # (the element itself counts as 0 among the rest of its column)
    same = outs[0] == outs[1]
    column = torch.zeros_like(hit)
    column[:, :, 1, :, col] = True
    assert same[~column].all() and same[column & ~hit].all() and hit.any()
    assert (torch.isnan(outs[1][hit]) if store == "fp8" else outs[1][hit] == float("-inf")).all()


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("B,n,Hq,Hkv,dh,top", [
    (50, 1, 12, 12, 64, 20), (100, 4, 12, 4, 128, 60), (65, 3, 16, 8, 64, 190), (400, 2, 2, 1, 128, 31), (33, 16, 8, 8, 128, 70), (37, 5, 21, 7, 128, 32),
    (60, 17, 8, 8, 128, 90), (90, 8, 12, 3, 64, 170), (300, 11, 2, 1, 64, 33)])
def test_many_short_caches(B, n, Hq, Hkv, dh, top, store):
    rng = np.random.default_rng(B + n + 2)
    check_call(rng, store, B, n, Hq, Hkv, dh, lengths(rng, B, top, "ragged"), spare=int(rng.integers(0, 3)) + 8 * (top < 31))


@pytest.mark.parametrize("store", ["fp8", "bf16", "fp32"])
def test_an_infinity_in_short_caches(store):
    """drafts see their own row alone among the new ones; every second sequence's second draft holds an infinity (fp8: NaN)"""
    rng = np.random.default_rng(12)
    B, n, H, dh = 60, 3, 8, 64
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    pos = [int(p) for p in rng.integers(0, 41, B)]
    (k, v, ks, vs), _ = cache_arrays(rng, store, (B, H, 64, dh))
    q = gpu(normal(rng, (B, n, H, dh), store != "fp32"), dt)
    c = F.make_kv_cache(k, v, ks, vs)
    bits, seq = torch.tensor([[1, 2, 4]] * B, dtype=torch.int64, device="cuda"), torch.tensor(pos, dtype=torch.int32, device="cuda")
    outs = []
    for spoil in (False, True):
        for b in range(0, B if spoil else 0, 2):
            if store == "fp8":
                v.view(torch.uint8)[b, :, pos[b] + 1, 9] = 0x7f
            else:
                v[b, :, pos[b] + 1, 9] = float("inf")
        out = torch.empty(B, n, H * dh, dtype=dt, device="cuda")
        F.forge_attn_tree(c, q, out, seq, max(pos), visible=bits, workspace=F.workspace(F.forge_attn_tree_workspace_bytes(c, H, n, max(pos))))
        outs.append(out.view(B, n, H, dh))
    hit = torch.zeros_like(outs[0], dtype=torch.bool)
    hit[::2, 1, :, 9] = True
    assert torch.equal(outs[0][~hit], outs[1][~hit])
    assert (torch.isnan(outs[1][hit]) if store == "fp8" else outs[1][hit] == float("inf")).all()
