"""Low-rank adapters of many requests on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2604_16498_amd import binding as F
from tree_inputs import gpu, normal
from util import host

pytestmark = pytest.mark.gpu


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def check(rng, M, K, ends, rank, n, ids, bf16, ldy=None, in_place=False, scaled=True, edit=None):
    dt, N = torch.bfloat16 if bf16 else torch.float32, ends[-1]
    x, base = normal(rng, (M, K), bf16), normal(rng, (M, ldy or N), bf16)
    a, b = normal(rng, (n, len(ends) * rank, K), bf16, K ** -0.5), normal(rng, (n, N, rank), bf16, 0.5)
    scale = rng.uniform(0.5, 2.0, n).astype(np.float32) if scaled else np.ones(n, np.float32)
    tx, tb, ta, tbb = gpu(x, dt), gpu(base, dt), gpu(a, dt), gpu(b, dt)
    if edit is not None:
        edit(tx, ta, tbb)
    d = F.make_adapters(ta, tbb, gpu(scale) if scaled else None, ends)
    y = tb if in_place else torch.full((M + 1, ldy or N), 7.0, dtype=dt, device="cuda")
    F.forge_adapters_add(d, tx, tb, y[:M], ints(ids), workspace=F.workspace(F.forge_adapters_workspace_bytes(d, M)))
    got = host(y[:M])
    if not in_place:
        assert (y[M] == 7.0).all() and (y[:, N:] == 7.0).all()       # what is not the output is left as it was
    else:
        np.testing.assert_array_equal(got[:, N:], base[:, N:])
    ref, first, second = O.adapters(x, base[:, :N], a, b, scale, ids, ends, rank)
    # products are exact or rounded once in fp32, sums of K (rank) terms off by K (rank) 2^-24 of their magnitude at most; bf16: the two halves of t
    # leave 2^-16 of it, and the output is rounded once
    off = first * (K + 4) * 2.0 ** -24 + second * ((rank + 8) * 2.0 ** -23 + (2.0 ** -16 if bf16 else 0.0)) + 2.0 ** -24 * np.abs(ref)
    off = off + (2.0 ** -8 * (np.abs(ref) + off) if bf16 else 2.0 ** -24 * np.abs(ref))
    err = np.abs(got[:, :N] - ref)
    assert (err <= off + 1e-30).all(), float((err / (off + 1e-30)).max())
    none = [m for m, i in enumerate(ids) if not 0 <= i < n]
    np.testing.assert_array_equal(got[none, :N], base[none, :N])
    return y[:M]


def runs(rng, M, n, requests):
    """adapters of rows: requests one after another, some without"""
    cuts = np.sort(rng.choice(M, min(M, requests) - 1, replace=False)) if min(M, requests) > 1 else []
    pick = rng.integers(-1, n, len(cuts) + 1)
    return [int(pick[np.searchsorted(cuts, m, side="left")]) for m in range(M)]


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M,K,ends,rank,n,requests", [
    (1, 64, [64], 8, 1, 1), (1, 8, [5], 8, 2, 1), (2, 768, [768], 8, 3, 2), (5, 72, [16, 48, 50], 16, 4, 5), (15, 520, [301], 24, 3, 4),
    (16, 256, [256], 40, 20, 16), (17, 1000, [64, 128, 192, 1001], 32, 5, 17), (33, 4096, [300], 64, 40, 33), (61, 2048, [512, 640, 768], 16, 61, 61),
    (100, 200, [900], 72, 3, 3), (130, 136, [96, 513], 128, 7, 9), (255, 320, [777], 96, 4, 30), (70, 4160, [66], 120, 2, 2)])
def test_adapters_of_a_batch(M, K, ends, rank, n, requests, bf16):
    rng = np.random.default_rng(M + K)
    check(rng, M, K, ends, rank, n, runs(rng, M, n, requests), bf16)


# 64 rows a block: whole ones, ends inside one, columns that are none of a block's 256, parts that end inside
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M,K,ends,rank,requests", [
    (1023, 128, [256], 16, 6), (1024, 128, [256], 16, 1), (1025, 136, [512], 8, 30), (1500, 72, [300], 64, 5), (1100, 1032, [256, 512, 768], 24, 3),
    (1088, 264, [272, 816, 900], 96, 17), (2050, 512, [1024], 128, 500)])
def test_adapters_of_prompts(M, K, ends, rank, requests, bf16):
    rng = np.random.default_rng(M + K)
    check(rng, M, K, ends, rank, 6, runs(rng, M, 6, requests), bf16)


# whole blocks of columns and rows that end inside a tile, in place and not, in the larger tiles and next to where they begin
@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M,K,ends,rank,requests", [
    (511, 72, [1536], 16, 4), (512, 72, [1536], 16, 4), (577, 264, [512, 1536], 64, 200), (703, 64, [1024], 8, 5), (704, 64, [1024], 8, 5),
    (513, 72, [1024, 2048, 2304], 64, 40), (899, 64, [2048], 8, 3), (900, 64, [2048], 8, 3), (1100, 64, [4096], 16, 300), (1025, 136, [2048], 16, 1), (1090, 72, [256, 768, 2048], 16, 400), (1100, 64, [4096], 24, 3), (2050, 64, [4096], 64, 9)])
def test_adapters_of_prompts_beside_whole_blocks(M, K, ends, rank, requests, bf16):
    rng = np.random.default_rng(M + K)
    ids = runs(rng, M, 6, requests)
    check(rng, M, K, ends, rank, 6, ids, bf16)
    check(rng, M, K, ends, rank, 6, ids, bf16, in_place=True)
    check(rng, M, K, ends, rank, 6, ids, bf16, ldy=ends[-1] + 8, in_place=True, scaled=False)


@pytest.mark.parametrize("bf16,rank", [(True, 128), (False, 72)])
def test_large_ranks_of_prompts(bf16, rank):
    rng = np.random.default_rng(rank)
    check(rng, 2570, 64, [4096], rank, 6, runs(rng, 2570, 6, 9), bf16, in_place=True)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M", [3, 40, 1030])
def test_in_place_strides_and_odd_addresses(M, bf16):
    rng = np.random.default_rng(M)
    for ldy in (None, 330, 331, 328):
        ids = runs(rng, M, 4, 7)
        check(rng, M, 96, [176, 325], 16, 4, ids, bf16, ldy=ldy, in_place=True, scaled=False)
        check(rng, M, 96, [176, 325], 16, 4, ids, bf16, ldy=ldy)


@pytest.mark.parametrize("M", [20, 1100])
def test_all_rows_of_one_adapter_and_of_none(M):
    rng = np.random.default_rng(M)
    for ids in ([2] * M, [-1] * M, [5] * M, [2**31 - 1] * M, [-2**31] * M, [m % 5 for m in range(M)]):
        check(rng, M, 128, [512], 16, 5, ids, True)
        check(rng, M, 128, [512], 16, 5, ids, True, in_place=True)


@pytest.mark.parametrize("M", [9, 1100])
def test_infinities_reach_the_rows_of_their_adapter_alone(M):
    """NaN and infinities in one adapter, and in the x of a row without one"""
    rng = np.random.default_rng(M)
    ids = [(m // 3) % 4 - 1 for m in range(M)]                # -1, 0, 1, 2, three rows each
    x, base = normal(rng, (M, 128)), normal(rng, (M, 320))
    a, b = normal(rng, (3, 8, 128)), normal(rng, (3, 320, 8))
    t = [gpu(z, torch.bfloat16) for z in (x, base, a, b)]
    call = lambda: F.forge_adapters_add(F.make_adapters(t[2], t[3]), t[0], t[1], torch.empty_like(t[1]), ints(ids),
                                        workspace=F.workspace(F.forge_adapters_workspace_bytes(F.make_adapters(t[2], t[3]), M)))
    clean = call()
    t[2][1, 3, 5] = float("inf")
    t[3][1, 100, 2] = float("nan")
    t[0][np.array([m for m in range(M) if ids[m] < 0])] = float("nan")
    dirty = call()
    rows = torch.tensor([i != 1 for i in ids], device="cuda")
    assert torch.equal(clean[rows], dirty[rows])
    assert torch.isnan(dirty[~rows][:, 100]).all() and not torch.isfinite(dirty[~rows]).any()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("M", [9, 1100])
def test_an_infinite_input_stays_infinite(M, bf16):
    """positive adapters: x = inf gives inf, -inf in another row -inf, not NaN"""
    rng = np.random.default_rng(M)
    dt = torch.bfloat16 if bf16 else torch.float32
    x, base, a, b = (gpu(z, dt) for z in (normal(rng, (M, 64)), normal(rng, (M, 320)), np.abs(normal(rng, (2, 16, 64))) + 0.1, np.abs(normal(rng, (2, 320, 16))) + 0.1))
    ids = [m % 2 for m in range(M)]
    d = F.make_adapters(a, b)
    call = lambda: F.forge_adapters_add(d, x, base, torch.empty_like(base), ints(ids), workspace=F.workspace(F.forge_adapters_workspace_bytes(d, M)))
    clean = call()
    x[3, 11], x[M - 1, 60] = float("inf"), -float("inf")
    got = call()
    assert (got[3] == float("inf")).all() and (got[M - 1] == -float("inf")).all()
    rest = [m for m in range(M) if m not in (3, M - 1)]
    assert torch.equal(got[rest], clean[rest])


def test_offsets_past_32_bits():
    """adapters more than 2^32 bytes into their tensors"""
    rng = np.random.default_rng(3)
    n, K, N, rank = 520, 65536, 48, 64
    a = torch.zeros(n, rank, K, dtype=torch.bfloat16, device="cuda")
    last = normal(rng, (rank, K), True, K ** -0.5)
    a[n - 1] = gpu(last, torch.bfloat16)
    b, x = normal(rng, (n, N, rank), True, 0.5), normal(rng, (3, K))
    d = F.make_adapters(a, gpu(b, torch.bfloat16))
    y = torch.zeros(3, N, dtype=torch.bfloat16, device="cuda")
    F.forge_adapters_add(d, gpu(x, torch.bfloat16), y, y, ints([n - 1, 0, n - 1]), workspace=F.workspace(F.forge_adapters_workspace_bytes(d, 3)))
    t = x.astype(np.float64) @ last.astype(np.float64).T
    ref = t @ b[n - 1].astype(np.float64).T
    ref[1] = 0.0
    first = (np.abs(x).astype(np.float64) @ np.abs(last).astype(np.float64).T) @ np.abs(b[n - 1]).astype(np.float64).T
    second = np.abs(t) @ np.abs(b[n - 1]).astype(np.float64).T
    off = first * (K + 4) * 2.0 ** -24 + second * 2.0 ** -15
    assert (np.abs(host(y) - ref) <= off + 2.0 ** -8 * (np.abs(ref) + off)).all() and (y[1] == 0).all()


@pytest.mark.parametrize("M", [12, 1200])
def test_two_graphs_share_a_workspace_and_another_stream(M):
    rng = np.random.default_rng(M)
    made = []
    for K, N, rank in ((256, 512, 16), (512, 300, 64)):
        t = [gpu(normal(rng, s, True, 0.3), torch.bfloat16) for s in ((M, K), (M, N), (4, rank, K), (4, N, rank))]
        made.append((F.make_adapters(t[2], t[3]), t[0], t[1], torch.empty_like(t[1]), ints(runs(rng, M, 4, 5))))
    ws = F.workspace(max(F.forge_adapters_workspace_bytes(m[0], M) for m in made))
    call = lambda m: F.forge_adapters_add(*m, workspace=ws)
    want = [call(m).clone() for m in made]
    graphs = []
    for m in made:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(m)
        graphs.append(g)
    side = torch.cuda.Stream()
    for _ in range(3):
        for m in made:
            m[3].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(m[3], w) for m, w in zip(made, want))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for m in made:
                call(m)
        side.synchronize()
        assert all(torch.equal(m[3], w) for m, w in zip(made, want))
    made[0][4].fill_(3)                        # adapters are read at replay
    graphs[0].replay()
    torch.cuda.synchronize()
    got = made[0][3].clone()
    assert torch.equal(got, call(made[0]))
