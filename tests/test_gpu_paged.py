"""A cache in pages on the GPU against the fp64 oracle: rows written and read back, attention of one new token per request."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from oracle import tree_oracle as T
from paper_2604_16498_amd import binding as F
from tree_inputs import cache_arrays, gpu, normal
from util import FP32_MAX_ABS, host

pytestmark = pytest.mark.gpu
HALF_ULP = 2.0 ** -8          # a bf16 rounding, relative
STORES = ["int8", "fp8", "bf16", "fp32"]


def ints(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def raw(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


# ---- rows ---------------------------------------------------------------------------------------


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("tokens,Hq,Hkv,dh,rot,style,P", [
    (1, 4, 4, 64, 64, "half", 16), (3, 8, 2, 128, 128, "half", 16), (37, 3, 3, 64, 16, "interleaved", 32), (70, 2, 1, 128, 96, "interleaved", 256),
    (300, 6, 2, 128, 32, "half", 64), (1100, 1, 1, 64, 64, "half", 1024)])
def test_append_and_read_back(tokens, Hq, Hkv, dh, rot, style, P, store):
    """Rows in slots of any order; some tokens without one.  Against forge_kv_append on one run of rows: the same bits; and against the oracle."""
    rng = np.random.default_rng(tokens + dh)
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    n_pages = -(-(tokens + 20) // P) + 2
    inc, factor = F.forge_rope_increments(10000.0, rot, scaling="ramp", by=8.0, context=8192.0, low=1.0, high=4.0)
    rope = F.make_rope_desc(inc.cuda(), style, factor)
    rows = normal(rng, (tokens, Hq + 2 * Hkv, dh), store != "fp32", std=3.0)
    t = gpu(rows, dt)
    q, k, v = t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:]
    positions = rng.integers(0, 30000, tokens)
    slots = rng.permutation(n_pages * P)[:tokens]
    left_out = rng.random(tokens) < 0.1
    slots[left_out] = rng.choice([-1, -2**31, n_pages * P, 2**31 - 1], int(left_out.sum()))
    (pk, pv, ks, vs), _ = cache_arrays(rng, store, (2, n_pages, Hkv, P, dh))
    before = [raw(x).clone() for x in (pk, pv, ks, vs) if x is not None]
    cache = F.make_paged_cache(pk, pv, ks, vs)
    q_out = torch.full((tokens, Hq, dh), 7.0, dtype=dt, device="cuda")
    F.forge_paged_append(cache, k, v, ints(slots), rope=rope, positions=ints(positions), q=q, q_out=q_out, layer=1)
    out = [torch.full((Hkv, tokens, dh), 7.0, dtype=dt, device="cuda").transpose(0, 1) for _ in range(2)]       # heads first, as a prompt takes them
    F.forge_paged_read(cache, *out, ints(slots), layer=1)
    # the same rows behind one another
    (fk, fv, fks, fvs), _ = cache_arrays(rng, store, (1, Hkv, tokens, dh))
    flat = F.make_kv_cache(fk, fv, fks, fvs)
    q_flat = torch.empty(1, tokens, Hq, dh, dtype=dt, device="cuda")
    F.forge_kv_append(flat, k[None], v[None], None, 0, rope=rope, positions=ints(positions)[None], q=q[None], q_out=q_flat)
    want = [torch.empty(1, Hkv, tokens, dh, dtype=dt, device="cuda") for _ in range(2)]
    F.forge_kv_read(flat, *want)
    there = torch.from_numpy(~left_out).cuda()
    assert torch.equal(q_out[there], q_flat[0][there]) and (q_out[~there] == 7.0).all()
    for got, w in zip(out, want):
        assert torch.equal(got[there], w[0].transpose(0, 1)[there]) and (got[~there] == 7.0).all()
    # pages: those rows hold the flat cache's, everything else is as it was
    layers = [x for x in (pk, pv, ks, vs) if x is not None]
    for old, new, one in zip(before, layers, [x for x in (fk, fv, fks, fvs) if x is not None]):
        want = old.clone()
        for i in np.flatnonzero(~left_out):
            want[1, slots[i] // P, :, slots[i] % P] = raw(one)[0, :, i]
        assert torch.equal(want, raw(new))
    # the oracle's rotation, to the code's half step
    theta, _ = T.frequencies(10000.0, rot, "ramp", 8.0, 8192.0, 1.0, 4.0)
    ref = T.rotate(rows[:, Hq:Hq + Hkv], positions[:, None], theta, style, factor)[~left_out]
    got = host(out[0])[~left_out]
    step = np.abs(ref).max(-1, keepdims=True) / T.TOP.get(store, np.inf)
    half = {"int8": 0.5 * step, "fp8": np.maximum(np.abs(ref) / 16, step * 2.0 ** -10)}.get(store, 0.0)
    top = np.abs(rows[:, Hq:Hq + Hkv]).max(-1, keepdims=True)[~left_out]
    turn = 2 * top * factor * (1.3e-7 + 2 * 2.0 ** -24)        # cos and sin, two products and a sum in fp32
    assert (np.abs(got - ref) <= turn + half * (1 + 1e-4) + (HALF_ULP if store != "fp32" else 2.0 ** -24) * (np.abs(ref) + half) + 1e-10).all()


@pytest.mark.parametrize("store", ["int8", "bf16"])
def test_append_in_place_without_rotation_and_slots_that_repeat_in_a_read(store):
    rng = np.random.default_rng(1)
    (k, v, ks, vs), _ = cache_arrays(rng, store, (3, 2, 16, 64))
    cache = F.make_paged_cache(k, v, ks, vs)
    t = gpu(normal(rng, (4, 5, 64)), torch.bfloat16)
    keep = t.clone()
    F.forge_paged_append(cache, t[:, 1:3], t[:, 3:], ints([47, 0, 16, 31]), q=t[:, :1], q_out=t[:, :1])
    assert torch.equal(t, keep)
    out = [torch.empty(6, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    F.forge_paged_read(cache, *out, ints([31, 31, 47, 0, 31, 16]))
    assert torch.equal(out[0][0], out[0][1]) and torch.equal(out[0][0], out[0][4])
    if store == "bf16":
        assert torch.equal(out[0][[3, 5, 0, 2]], t[[1, 2, 3, 0], 1:3]) and torch.equal(out[1][2], t[0, 3:])


def test_empty_slots_write_nothing():
    (k, v, ks, vs), _ = cache_arrays(np.random.default_rng(2), "int8", (2, 1, 16, 64))
    before = k.clone()
    t = torch.ones(300, 1, 64, dtype=torch.bfloat16, device="cuda")
    F.forge_paged_append(F.make_paged_cache(k, v, ks, vs), t, t, ints([-1] * 300))
    assert torch.equal(k, before)


# ---- attention ----------------------------------------------------------------------------------


def tables(rng, lengths, P, cols, n_pages, bad=-1):
    order = list(rng.permutation(n_pages))
    table = np.full((len(lengths), cols), bad, np.int64)
    for b, n in enumerate(lengths):
        for c in range(-(-max(n, 0) // P)):
            table[b, c] = order.pop()
    return table


def attention_bound(store, group, ref, mag):
    """bf16: the output's rounding, 2^-8 of it, and the weights', of sum P |v|: 2^-16 where up to 8 heads share a cache head, else
    2^-8; fp32 scores add about 1e-5 of it."""
    if store == "fp32":
        return FP32_MAX_ABS
    return HALF_ULP * np.abs(ref) + ((2.0 ** -16 if group <= 8 else HALF_ULP) * 1.02 + 2e-5) * 1.01 * mag + 1e-6


def attend(rng, store, lengths, Hq, Hkv, dh, P, most=None, extra=2, bad=-1, q=None, cache=None, table=None, edit=None, scale=None):
    B, most = len(lengths), most or max(1, max(lengths))
    cols = -(-most // P) + extra
    n_pages = sum(-(-max(n, 0) // P) for n in lengths) + 3
    table = tables(rng, lengths, P, cols, n_pages, bad) if table is None else table
    (k, v, ks, vs), (rk, rv) = cache if cache is not None else cache_arrays(rng, store, (n_pages, Hkv, P, dh))
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    q = normal(rng, (B, Hq, dh), store != "fp32") if q is None else q
    if edit is not None:
        edit(k, v, ks, vs, table)
    c = F.make_paged_cache(k, v, ks, vs)
    ws = F.workspace(F.forge_attn_paged_workspace_bytes(c, Hq, B, most))
    out = torch.full((B + 1, Hq * dh), 7.0, dtype=dt, device="cuda")
    scale = dh ** -0.5 if scale is None else scale
    F.forge_attn_paged(c, gpu(q, dt), out[:B], ints(lengths), ints(table), most, scale=scale, workspace=ws)
    ref, mag = O.attention(q, rk, rv, table, lengths, scale)
    got = host(out[:B]).reshape(ref.shape)
    assert np.isfinite(got).all() and (out[B] == 7.0).all()
    bound = attention_bound(store, Hq // Hkv, ref, mag)
    err = np.abs(got - ref)
    assert (err <= bound).all(), (err / (mag + 1e-30)).max()
    return out[:B]


# lengths around tiles of 32, halves of 16, units of 128, what is cut from 512 rows on; groups of 1 to 40 query heads; idle requests
@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("lengths,Hq,Hkv,dh,P", [
    ([1], 1, 1, 64, 16), ([0], 4, 2, 128, 16), ([0, 0, 0], 8, 8, 64, 32), ([2, 15, 16, 17], 4, 4, 128, 16), ([31, 32, 33, 0, 1], 12, 12, 64, 16),
    ([127, 128, 129], 32, 8, 128, 32), ([511, 512, 513, 0], 8, 2, 64, 16), ([700], 16, 1, 128, 64), ([1, 3000], 17, 1, 64, 128),
    ([4000, 0, 5], 40, 1, 128, 256), ([0, 2500, 0, 0, 1300, 0], 6, 2, 128, 16), ([9001], 8, 2, 128, 1024), ([5000, 4999], 33, 3, 64, 512)])
def test_attention_over_pages(lengths, Hq, Hkv, dh, P, store):
    attend(np.random.default_rng(sum(lengths) + Hq), store, lengths, Hq, Hkv, dh, P)


@pytest.mark.parametrize("store", ["int8", "bf16"])
@pytest.mark.parametrize("batch,top,Hkv,dh", [(70, 90, 12, 64), (65, 200, 8, 128), (257, 40, 2, 64), (300, 700, 1, 64), (20, 900, 2, 128), (64, 600, 3, 64)])
def test_many_requests(batch, top, Hkv, dh, store):
    """a wave a pair, whole pairs by length, dealt ones, and batches past what is dealt; a third of them idle"""
    rng = np.random.default_rng(batch)
    lengths = [0 if rng.random() < 0.3 else int(rng.integers(1, top + 1)) for _ in range(batch)]
    lengths[-1] = 0
    lengths[batch // 2] = top
    attend(rng, store, lengths, 2 * Hkv, Hkv, dh, 16)


@pytest.mark.parametrize("store", STORES)
def test_a_bound_above_the_lengths_and_lengths_outside(store):
    """max_len far above what there is: the cut changes, the result not by more than rounding; lengths are clamped"""
    rng = np.random.default_rng(7)
    attend(rng, store, [40, 0, 300], 8, 2, 64, 16, most=5000)
    attend(rng, store, [1, 0, 2], 4, 1, 128, 32, most=100000)
    q, cache = normal(rng, (2, 4, 64), store != "fp32"), cache_arrays(rng, store, (9, 2, 16, 64))
    table = np.array([[0, 1, 2, 3], [4, 5, 6, 7]])
    want = attend(rng, store, [64, 0], 4, 2, 64, 16, q=q, cache=cache, table=table)
    c = F.make_paged_cache(*cache[0])
    out = torch.empty_like(want)
    F.forge_attn_paged(c, gpu(q, want.dtype), out, ints([10**6, -9]), ints(table), 64)
    assert torch.equal(out, want)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dh,lengths,P", [(64, [37, 1, 0], 16), (128, [37, 16, 700], 64), (64, [1025, 3], 128)])
def test_what_lies_behind_a_length_does_not_reach_it(store, dh, lengths, P):
    """Infinities and NaN in the rest of a last page, in free pages, and behind table entries that are not used"""
    rng = np.random.default_rng(4)
    n_pages = sum(-(-n // P) for n in lengths) + 3
    q, cache = normal(rng, (len(lengths), 4, dh), store != "fp32"), cache_arrays(rng, store, (n_pages, 2, P, dh))
    table = tables(rng, lengths, P, -(-max(lengths) // P) + 2, n_pages)
    clean = attend(rng, store, lengths, 4, 2, dh, P, q=q, cache=cache, table=table)

    def spoil(k, v, ks, vs, table):
        used = np.zeros((n_pages, P), bool)
        for b, n in enumerate(lengths):
            for r in range(n):
                used[table[b, r // P], r % P] = True
        for i, (page, r) in enumerate(zip(*np.nonzero(~used))):
            x = (float("nan"), float("inf"), float("-inf"))[i % 3]
            if ks is not None:
                ks[page, :, r] = x
                vs[page, :, r] = x
            if store == "fp8":
                v.view(torch.uint8)[page, :, r] = 0x7f
                k.view(torch.uint8)[page, :, r] = 0xff
            elif store != "int8":
                k[page, :, r] = x
                v[page, :, r] = x
    spoilt = [None if t is None else t.clone() for t in cache[0]]
    spoil(*spoilt, table)
    c, out = F.make_paged_cache(*spoilt), torch.empty_like(clean)
    ws = F.workspace(F.forge_attn_paged_workspace_bytes(c, 4, len(lengths), max(lengths)))
    free = int(np.setdiff1d(np.arange(n_pages), table)[0])
    for rest in (-1, 10**9, -2**31, free):                    # what unused entries say
        F.forge_attn_paged(c, gpu(q, clean.dtype), out, ints(lengths), ints(np.where(table < 0, rest, table)), max(lengths), workspace=ws)
        assert torch.equal(out, clean)


def test_what_lies_in_a_row_reaches_its_request_alone():
    rng = np.random.default_rng(5)
    q, cache = normal(rng, (2, 2, 64)), cache_arrays(rng, "bf16", (8, 1, 16, 64))
    table = np.array([[0, 1, 2], [3, 4, 5]])
    clean = attend(rng, "bf16", [40, 40], 2, 1, 64, 16, q=q, cache=cache, table=table)
    cache[0][1][4, 0, 3, 7] = float("inf")
    out = torch.empty_like(clean)
    F.forge_attn_paged(F.make_paged_cache(*cache[0]), gpu(q, torch.bfloat16), out, ints([40, 40]), ints(table), 40)
    assert torch.equal(out[0], clean[0]) and (out[1].view(2, 64)[:, 7] == float("inf")).all()
    out = out[1].view(2, 64)
    assert torch.equal(out[:, :7], clean[1].view(2, 64)[:, :7]) and torch.equal(out[:, 8:], clean[1].view(2, 64)[:, 8:])


@pytest.mark.parametrize("store", ["int8", "bf16"])
def test_large_scores(store):
    """one row dominates by far, late in the request: the running maximum has to move; and all scores alike; and far apart between shares"""
    rng = np.random.default_rng(6)
    q = normal(rng, (1, 4, 64))
    tensors, values = cache_arrays(rng, store, (60, 1, 16, 64))
    table = rng.permutation(60)[None]
    page, r = table[0, 777 // 16], 777 % 16
    tensors[0][page, 0, r] = gpu(np.sign(q[0, 2]) * (127 if store == "int8" else 90.0)).to(tensors[0].dtype)
    values[0][page, 0, r] = host(tensors[0][page, 0, r]) * (1.0 if store != "int8" else float(tensors[2][page, 0, r]))
    for x in (q, np.zeros_like(q)):
        attend(rng, store, [890], 4, 1, 64, 16, q=x, cache=(tensors, values), table=table)


@pytest.mark.parametrize("store", ["int8", "bf16", "fp32"])
def test_pages_shared_by_requests_and_a_layer_of_several(store):
    rng = np.random.default_rng(8)
    L, n_pages, Hkv, P, dh = 3, 12, 2, 16, 64
    (k, v, ks, vs), (rk, rv) = cache_arrays(rng, store, (L, n_pages, Hkv, P, dh))
    c = F.make_paged_cache(k, v, ks, vs)
    table, lengths = np.array([[3, 5, 1, 0], [3, 5, 9, 8], [3, 5, 1, 2]]), [50, 64, 33]
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    q = normal(rng, (3, 7, dh), store != "fp32")
    for layer in range(L):
        out = torch.empty(3, 4 * dh, dtype=dt, device="cuda")
        F.forge_attn_paged(c, gpu(q, dt)[:, 2:6], out, ints(lengths), ints(table), 64, layer=layer)
        ref, mag = O.attention(q[:, 2:6], rk[layer], rv[layer], table, lengths, dh ** -0.5)
        assert (np.abs(host(out).reshape(ref.shape) - ref) <= attention_bound(store, 2, ref, mag)).all()


@pytest.mark.parametrize("store", ["int8", "bf16"])
def test_offsets_past_32_bits_and_strides(store):
    """pages more than 2^32 bytes apart, heads with room between them"""
    rng = np.random.default_rng(9)
    dh, P, Hkv, n = 64, 16, 2, 4
    far = ((1 << 32) // (1 if store == "int8" else 2) // (n - 1) // dh + 4096) * dh
    size, hs = far * (n - 1) + 2 * (P + 8) * dh, (P + 8) * dh
    dt = torch.int8 if store == "int8" else torch.bfloat16
    (k, v, ks, vs), (rk, rv) = cache_arrays(rng, store, (n, Hkv, P, dh))
    big = [torch.empty(size, dtype=dt, device="cuda").as_strided((n, Hkv, P, dh), (far, hs, dh, 1)) for _ in range(2)]
    scales = [None, None]
    if store == "int8":
        scales = [torch.empty(size // dh, device="cuda").as_strided((n, Hkv, P), (far // dh, P + 8, 1)) for _ in range(2)]
        scales[0].copy_(ks)
        scales[1].copy_(vs)
    big[0].copy_(k)
    big[1].copy_(v)
    c, out = F.make_paged_cache(*big, *scales), torch.empty(1, 4 * dh, dtype=torch.bfloat16, device="cuda")
    table, q = np.array([[3, 0, 2, 1]]), normal(rng, (1, 4, dh))
    F.forge_attn_paged(c, gpu(q, torch.bfloat16), out, ints([61]), ints(table), 64)
    ref, mag = O.attention(q, rk, rv, table, [61], dh ** -0.5)
    assert (np.abs(host(out).reshape(ref.shape) - ref) <= attention_bound(store, 2, ref, mag)).all()
    new = gpu(normal(rng, (2, 2, dh)), torch.bfloat16)
    F.forge_paged_append(c, new, new, ints([3 * P + 5, 2 * P + 1]))
    back = [torch.empty(2, 2, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    F.forge_paged_read(c, *back, ints([3 * P + 5, 2 * P + 1]))
    assert (back[0].float() - new.float()).abs().max() <= 0.02 and torch.equal(*back)


def test_two_graphs_share_a_workspace_and_another_stream():
    """the same bits every run; two captured calls of different sizes replayed in turn over one workspace"""
    rng = np.random.default_rng(10)
    made = []
    for store, lengths, P in (("int8", [2900, 0, 1234], 16), ("bf16", [3000] * 2, 64)):
        cache = cache_arrays(rng, store, (sum(-(-n // P) for n in lengths) + 3, 2, P, 128))
        table = tables(rng, lengths, P, 200, cache[0][0].shape[0])
        q = gpu(normal(rng, (len(lengths), 8, 128)), torch.bfloat16)
        made.append((F.make_paged_cache(*cache[0]), q, torch.empty(len(lengths), 8 * 128, dtype=torch.bfloat16, device="cuda"), ints(lengths), ints(table)))
    ws = F.workspace(max(F.forge_attn_paged_workspace_bytes(c, 8, q.shape[0], 3000) for c, q, *_ in made))
    call = lambda m: F.forge_attn_paged(m[0], m[1], m[2], m[3], m[4], 3000, workspace=ws)
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
            m[2].zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(m[2], w) for m, w in zip(made, want))
        for m, w in zip(made, want):
            m[2].zero_()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                call(m)
            side.synchronize()
            assert torch.equal(m[2], w)
    # lengths are read at replay
    made[0][3].copy_(ints([1, 2900, 0]))
    made[0][4].copy_(made[0][4][[2, 0, 1]])
    graphs[0].replay()
    torch.cuda.synchronize()
    got = made[0][2].clone()
    call(made[0])
    assert torch.equal(got, made[0][2]) and (got[2] == 0).all()
