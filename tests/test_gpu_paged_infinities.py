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
