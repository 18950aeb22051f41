"""Infinities in rows of v that a request sees, in attention over pages: they come out as the formula has them, whatever the cache's type and
however the rows are cut."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2604_16498_amd import binding as F
from test_gpu_paged import ints, tables
from tree_inputs import cache_arrays, gpu, normal
from util import host

pytestmark = pytest.mark.gpu


def attend(cache, q, lengths, table, dt=torch.bfloat16):
    B, Hq, dh = q.shape
    c, most = F.make_paged_cache(*cache), max(lengths)
    out = torch.empty(B, Hq * dh, dtype=dt, device="cuda")
    F.forge_attn_paged(c, gpu(q, dt), out, ints(lengths), ints(table), most,
                       workspace=F.workspace(F.forge_attn_paged_workspace_bytes(c, Hq, B, most)))
    return host(out).reshape(q.shape)


# whole pairs, a wave a pair, shares; up to 8, 9 to 16 and more query heads a cache head
@pytest.mark.parametrize("store", ["int8", "fp8"])
@pytest.mark.parametrize("lengths,Hq,Hkv,dh,P", [([40, 7], 2, 1, 64, 16), ([40, 7], 12, 1, 128, 16), ([300, 44], 40, 2, 64, 64), ([2500, 700], 8, 2, 128, 32),
                                                 ([3000, 1], 20, 1, 64, 64), ([60] * 130, 16, 8, 64, 16), ([60] * 130, 10, 5, 128, 16)])
def test_an_infinite_scale(lengths, Hq, Hkv, dh, P, store):
    """A row of the first request has it: each element infinite as its code says, NaN where the code is 0"""
    rng = np.random.default_rng(sum(lengths) + Hq)
    n_pages = sum(-(-n // P) for n in lengths) + 3
    table = tables(rng, lengths, P, -(-max(lengths) // P) + 1, n_pages)
    tensors, values = cache_arrays(rng, store, (n_pages, Hkv, P, dh))
    q = normal(rng, (len(lengths), Hq, dh))
    clean = attend(tensors, q, lengths, table)
    row = lengths[0] // 2
    page, r = table[0, row // P], row % P
    tensors[3][page, :, r] = float("inf")
    v = values[1].copy()
    with np.errstate(invalid="ignore"):
        v[page, :, r] *= np.inf
        ref, _ = O.attention(q[:1], values[0], v, table, lengths[:1], dh ** -0.5)
    got = attend(tensors, q, lengths, table)
    assert not np.isfinite(ref).any() and np.isinf(ref).any()
    np.testing.assert_array_equal(got[:1], ref)              # (NaN equal to NaN here)
    np.testing.assert_array_equal(got[1:], clean[1:])


CUTS = [  # rows of every request, requests, query heads, cache heads, head size, page; the loud row and the one with an infinity
    # in one tile, in tiles of two waves, in two tiles of one wave: either first
    ([20], 1, 2, 1, 64, 16, 3, 15), ([20], 1, 12, 1, 128, 16, 15, 3), ([300], 1, 4, 1, 64, 32, 5, 40), ([300], 1, 20, 1, 128, 16, 40, 5),
    ([300], 1, 12, 2, 64, 16, 5, 133), ([300], 1, 2, 1, 128, 64, 290, 161), ([300], 1, 8, 1, 64, 16, 133, 5),
    # shares
    ([5000], 1, 8, 2, 64, 16, 10, 4990), ([5000], 1, 9, 1, 128, 64, 4990, 10), ([5000], 1, 2, 1, 64, 16, 2600, 2601), ([5000, 3, 5000], 3, 24, 1, 64, 128, 2000, 2900),
    # a wave a pair
    ([60], 130, 8, 8, 64, 16, 2, 59), ([60], 130, 45, 5, 128, 16, 50, 7)]


@pytest.mark.parametrize("store", ["bf16", "fp32", "int8", "fp8"])
@pytest.mark.parametrize("lengths,B,Hq,Hkv,dh,P,loud,odd", CUTS)
@pytest.mark.parametrize("score", [40.0, 11.5])
def test_an_infinity_of_tiny_weight(lengths, B, Hq, Hkv, dh, P, loud, odd, score, store):
    """One row outweighs all others: e^-320 (e^-92, 2^-133 and below) and more is left to them, 0 in fp32 (subnormal), but positive.  So an
    infinity among them reaches the output, and nothing else does."""
    rng = np.random.default_rng(loud + odd)
    lengths = lengths * (B // len(lengths))
    n_pages = sum(-(-n // P) for n in lengths) + 3
    table = tables(rng, lengths, P, -(-max(lengths) // P) + 1, n_pages)
    (k, v, ks, vs), (_, rv) = cache_arrays(rng, store, (n_pages, Hkv, P, dh))
    want = np.zeros((B, Hq, dh))
    (k if ks is None else k.view(torch.uint8)).zero_()
    if ks is not None:
        ks.fill_(1.0)
    tall = [b for b, n in enumerate(lengths) if n > max(loud, odd)]
    pages, rows = (torch.tensor([[f(b, r) for b in tall] for r in (loud, odd)], device="cuda")
                   for f in (lambda b, r: int(table[b, r // P]), lambda b, r: r % P))
    if ks is None:
        k[pages[0], :, rows[0]] = score                              # q of ones: a score of `score` sqrt(dh) against 0
    else:
        k.view(torch.uint8)[pages[0], :, rows[0]] = 1 if store == "int8" else 0x38       # the code of 1
    if ks is not None:
        ks[pages[0], :, rows[0]] = score
        vs[pages[1], :, rows[1]] = float("inf")
    else:
        v[pages[1], :, rows[1], 5] = float("inf")
        v[pages[1], Hkv - 1, rows[1], 6] = -float("inf")
    for b in tall:
        want[b] = np.repeat(rv[table[b, loud // P], :, loud % P], Hq // Hkv, 0)
        if ks is None:
            want[b, :, 5] = np.inf
            want[b, -(Hq // Hkv):, 6] = -np.inf
        else:                          # a code times an infinity, NaN where it is 0
            with np.errstate(invalid="ignore"):
                want[b] = np.repeat(rv[table[b, odd // P], :, odd % P], Hq // Hkv, 0) * np.inf
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    got = attend([k, v, ks, vs], np.ones((B, Hq, dh), np.float32), lengths, table, dt)[tall]
    want = want[tall]
    # finite elements: a weight of 1 (in bf16 exactly), the others' share and the fp32 divisions below 2^-22, then a rounding
    odd_ones = ~np.isfinite(want)
    np.testing.assert_array_equal(np.where(odd_ones, got, 0.0), np.where(odd_ones, want, 0.0))
    off = np.abs(np.where(odd_ones, 0.0, got - np.where(odd_ones, 0.0, want)))
    assert (off <= (2.0 ** -22 + (2.0 ** -8 if store != "fp32" else 0.0)) * np.abs(np.where(odd_ones, 0.0, want)) + 1e-30).all()


@pytest.mark.parametrize("store", ["bf16", "int8"])
def test_nan_stays_nan_beside_a_far_maximum(store):
    """A NaN in a row of k that counts for nothing beside another's score, and one in v: the request's whole output, and its column"""
    rng = np.random.default_rng(3)
    table = rng.permutation(20)[None]
    (k, v, ks, vs), _ = cache_arrays(rng, store, (20, 1, 16, 64))
    k.zero_()
    page, r = int(table[0, 3]), 9
    if ks is None:
        k[page, 0, r] = 40.0
    else:
        ks.fill_(1.0)
        k[page, 0, r] = 1
        ks[page, 0, r] = 40.0
    q = np.ones((1, 2, 64), np.float32)
    at = int(table[0, 10]), 0, 4
    if ks is None:
        v[(*at, 7)] = float("nan")
        got = attend([k, v, ks, vs], q, [300], table)
        assert np.isnan(got[..., 7]).all() and np.isfinite(np.delete(got, 7, -1)).all()
        k[(*at, 1)] = float("nan")
    else:
        ks[at] = float("nan")
    assert np.isnan(attend([k, v, ks, vs], q, [300], table)).all()
