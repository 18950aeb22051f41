"""The host side of serving many requests over one pool of pages: refusals, workspace sizes, pins of the oracle."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2604_16498_amd import binding as B


def _cache(**kw):
    c = B.PagedCache()
    c.type, c.dt, c.n_layers, c.n_pages, c.page_rows, c.kv_heads, c.head_dim = 1, 1, 1, 100, 16, 4, 64
    c.head_stride, c.page_stride, c.layer_stride = 16 * 64, 4 * 16 * 64, 0
    c.k, c.v, c.k_scale, c.v_scale = 0x10000, 0x20000, 0x30000, 0x40000
    for name, v in kw.items():
        setattr(c, name, v)
    return c


def _heads(ptr=0x50000, bs=1024, ts=1024, hs=64):
    return B.Heads(ptr, bs, ts, hs)


BAD_CACHES = [(dict(k=None), 1), (dict(k=0x10004), 1), (dict(v=0x10000), 1), (dict(type=3), 1), (dict(dt=2), 1), (dict(dt=0), 2),
              (dict(head_dim=96), 2), (dict(n_pages=0), 1), (dict(kv_heads=0), 1), (dict(page_rows=0), 1), (dict(page_rows=8), 2),
              (dict(page_rows=48), 2), (dict(page_rows=2048), 2), (dict(n_layers=0), 1), (dict(k_scale=None), 1),
              (dict(v_scale=0x30000), 1), (dict(k_scale=0x30002), 1), (dict(head_stride=64), 1), (dict(head_stride=16 * 64 + 8), 1),
              (dict(page_stride=4 * 16 * 64 + 32), 1), (dict(page_stride=64), 1), (dict(page_stride=1 << 41), 1), (dict(n_pages=1 << 27), 2),
              (dict(kv_heads=40000), 2), (dict(n_layers=2, layer_stride=0), 1)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_a_bad_cache_is_refused_everywhere(bad, status):
    l, c, ref = B.lib(), _cache(**bad), C.byref
    x, y, p = _heads(), _heads(0x90000), C.c_void_p(0x70000)
    assert l.forge_paged_append(ref(c), 0, None, ref(x), ref(x), None, None, 0, p, None, 3, None) == status
    assert l.forge_paged_read(ref(c), 0, ref(x), ref(y), p, 3, None) == status
    assert l.forge_attn_paged(ref(c), 0, ref(x), p, p, p, 4, 4, 2, 10, 0.1, None, 0, None) == status
    assert l.forge_attn_paged_workspace_bytes(ref(c), 4, 2, 10000) == 0


def test_refusals_of_rows_and_attention():
    l, ref, vp = B.lib(), C.byref, C.c_void_p
    c, x, p = _cache(), _heads(), vp(0x70000)
    attn = lambda layer=0, q=x, out=p, lens=p, table=p, cols=4, hq=8, batch=3, most=64, scale=0.1: l.forge_attn_paged(
        ref(c), layer, ref(q), out, lens, table, cols, hq, batch, most, scale, None, 0, None)
    for kw, status in ((dict(layer=1), 1), (dict(layer=-1), 1), (dict(hq=6), 1), (dict(hq=0), 1), (dict(batch=0), 1), (dict(most=0), 1),
                       (dict(most=65), 1), (dict(cols=0), 1), (dict(most=-5), 1), (dict(scale=0.0), 1), (dict(scale=math.nan), 1),
                       (dict(out=None), 1), (dict(out=vp(0x70008)), 1), (dict(out=vp(0x50000)), 1), (dict(out=vp(0x10000)), 1),
                       (dict(lens=None), 1), (dict(lens=vp(0x70002)), 1), (dict(table=None), 1), (dict(table=vp(0x70001)), 1),
                       (dict(q=_heads(ptr=0)), 1), (dict(q=_heads(ptr=0x50008)), 1), (dict(q=_heads(bs=1028)), 1), (dict(q=_heads(hs=-64)), 1),
                       (dict(hq=80000), 2), (dict(batch=70000), 2), (dict(cols=1 << 27, most=10), 2), (dict(cols=(1 << 27) - 1, most=(1 << 30) + 1), 2)):
        assert attn(**kw) == status, kw
    assert attn(cols=1000, most=16000) == 3                              # its shares need a workspace
    app = lambda r=None, k=x, v=x, q=None, qo=None, hq=0, slots=p, pos=None, n=4, layer=0: l.forge_paged_append(
        ref(c), layer, r, ref(k), ref(v), q, qo, hq, slots, pos, n, None)
    rope = B.RopeDesc(64, 0, 1.0, 0x60000)
    for kw, status in ((dict(k=_heads(ptr=0)), 1), (dict(v=_heads(ts=4)), 1), (dict(n=0), 1), (dict(layer=3), 1), (dict(slots=None), 1),
                       (dict(slots=vp(0x70002)), 1), (dict(pos=vp(0x70002)), 1), (dict(r=ref(rope)), 1),      # a rotation without positions
                       (dict(r=ref(B.RopeDesc(128, 0, 1.0, 0x60000)), pos=p), 1), (dict(r=ref(B.RopeDesc(24, 0, 1.0, 0x60000)), pos=p), 2),
                       (dict(q=ref(x), qo=None, hq=4), 1), (dict(q=ref(x), qo=ref(x), hq=0), 1), (dict(k=_heads(ptr=0x10000)), 1),
                       (dict(q=ref(x), qo=ref(_heads(hs=128)), hq=4), 1), (dict(q=ref(x), qo=ref(_heads(ptr=0x20000)), hq=4), 1),
                       (dict(n=(1 << 24) + 1), 2), (dict(q=ref(x), qo=ref(_heads(0x90000, hs=0)), hq=4), 1)):
        assert app(**kw) == status, kw
    read = lambda k=x, v=_heads(0x90000), slots=p, n=4, layer=0: l.forge_paged_read(ref(c), layer, ref(k), ref(v), slots, n, None)
    for kw, status in ((dict(k=_heads(0x90000)), 1), (dict(v=_heads(0x10000)), 1), (dict(slots=None), 1), (dict(n=0), 1), (dict(layer=1), 1),
                       (dict(k=_heads(ts=0)), 1), (dict(k=_heads(hs=32)), 1), (dict(n=(1 << 24) + 1), 2)):
        assert read(**kw) == status, kw


def test_refusals_of_the_bookkeeping():
    l, ref, vp = B.lib(), C.byref, C.c_void_p
    names = ("lengths", "change", "out", "granted", "starts", "slots", "positions", "owners")
    good = {n: 0x1000 * (i + 1) for i, n in enumerate(names)}
    pool = dict(n_pages=10, page_rows=16, batch=3, table_cols=4, free_pages=0x100000, free_count=0x200000, table=0x300000)

    def call(tokens=5, change_pool={}, **kw):
        p = B.PagePool(*[{**pool, **change_pool}[n] for n in ("n_pages", "page_rows", "batch", "table_cols", "free_pages", "free_count", "table")])
        a = {**good, **kw}
        return l.forge_pages_assign(ref(p), *[None if a[n] is None else vp(a[n]) for n in names], tokens, None)
    for kw, status in ([(dict(change_pool={n: 0}), 1) for n in ("n_pages", "page_rows", "batch", "table_cols")] +
                       [(dict(change_pool={n: None}), 1) for n in ("free_pages", "free_count", "table")] +
                       [(dict(change_pool={n: 0x100002}), 1) for n in ("free_pages", "free_count", "table")] +
                       [({n: None}, 1) for n in names] + [({n: 0x900001}, 1) for n in names] +
                       [(dict(tokens=-1), 1), (dict(tokens=(1 << 24) + 1), 2), (dict(change_pool=dict(page_rows=20)), 2),
                        (dict(change_pool=dict(page_rows=8)), 2), (dict(change_pool=dict(batch=70000)), 2),
                        (dict(change_pool=dict(n_pages=1 << 26)), 2), (dict(change_pool=dict(table_cols=(1 << 25) + 1)), 2),
                        (dict(change_pool=dict(n_pages=1 << 25, page_rows=64)), 2),
                        # the same memory twice
                        (dict(granted=good["lengths"]), 1), (dict(out=good["change"]), 1), (dict(granted=good["out"]), 1),
                        (dict(starts=good["granted"]), 1), (dict(slots=good["positions"]), 1), (dict(slots=good["owners"]), 1),
                        (dict(owners=good["change"]), 1), (dict(positions=good["lengths"]), 1), (dict(slots=0x300000), 1),
                        (dict(granted=0x100000), 1), (dict(change=0x300000), 1)]):
        assert call(**kw) == status, kw


def test_refusals_of_the_adapters():
    l, ref, vp = B.lib(), C.byref, C.c_void_p

    def desc(**kw):
        d = B.Adapters(1, 5, 16, 64, 96, 2, (C.c_int * 4)(32, 96, 0, 0), 0x10000, 0x20000, 0x30000)
        for n, v in kw.items():
            setattr(d, n, (C.c_int * 4)(*v) if n == "part_end" else v)
        return d
    call = lambda x=0x40000, base=0x50000, y=0x60000, ids=0x70000, M=7, ldy=0, ws=0x80000, nb=1 << 30, **kw: l.forge_adapters_add(
        ref(desc(**kw)), *[None if p is None else vp(p) for p in (x, base, y, ids)], M, ldy, vp(ws) if ws else None, nb, None)
    for kw, status in ((dict(x=None), 1), (dict(base=None), 1), (dict(y=None), 1), (dict(ids=None), 1), (dict(x=0x40008), 1),
                       (dict(ids=0x70002), 1), (dict(y=0x40000), 1), (dict(M=0), 1), (dict(ldy=95), 1), (dict(ws=0x80004), 1),
                       (dict(ws=0, nb=0), 3), (dict(nb=100), 3), (dict(dt=2), 1), (dict(a=None), 1), (dict(b=0x20004), 1),
                       (dict(scale=0x30002), 1), (dict(n_adapters=0), 1), (dict(rank=0), 1), (dict(rank=12), 2), (dict(rank=136), 2),
                       (dict(K=60), 2), (dict(K=0), 1), (dict(dt=0, K=62), 2), (dict(n_parts=0), 1), (dict(n_parts=5), 2),
                       (dict(part_end=(32, 95, 0, 0)), 1), (dict(part_end=(40, 96, 0, 0)), 2), (dict(part_end=(96, 96, 0, 0)), 1),
                       (dict(part_end=(0, 96, 0, 0)), 1), (dict(M=(1 << 24) + 1), 2), (dict(M=1 << 22, N=1 << 20, part_end=(32, 1 << 20, 0, 0)), 2)):
        assert call(**kw) == status, kw
    assert l.forge_adapters_workspace_bytes(ref(desc(rank=12)), 4) == 0 and l.forge_adapters_workspace_bytes(ref(desc()), 0) == 0


def test_workspace_of_the_attention_serves_every_smaller_call():
    for hq, hkv in ((8, 2), (12, 12), (32, 8), (40, 1)):
        c = _cache(kv_heads=hkv, n_pages=1 << 20, page_stride=hkv * 16 * 64)
        sizes = [[B.forge_attn_paged_workspace_bytes(c, hq, b, n) for n in (1, 100, 512, 513, 700, 2000, 9000, 10**6)]
                 for b in (1, 2, 7, 64, 255, 256, 257, 5000)]
        assert (np.diff(sizes, axis=0) >= 0).all() and (np.diff(sizes, axis=1) >= 0).all()


@pytest.mark.parametrize("dt", [0, 1])
def test_workspace_of_the_adapters_serves_every_smaller_call(dt):
    for K, N, rank, parts in ((768, 768, 8, 1), (4096, 6144, 16, 3), (4096, 4096, 64, 1), (64, 512, 128, 2), (14336, 4096, 40, 1)):
        d = B.Adapters(dt, 4, rank, K, N, parts, (C.c_int * 4)(*([64, 128][:parts - 1] + [N])), 0x10000, 0x20000, None)
        sizes = [B.forge_adapters_workspace_bytes(d, m) for m in list(range(1, 1200)) + [2000, 4096, 100000]]
        assert (np.diff(sizes) >= 0).all() and sizes[0] >= parts * rank * 4


def test_binding_refuses_what_it_cannot_pass_on():
    t = torch.zeros(4, 8, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.make_page_pool(t[0], t[0, :1], t, 16)                # not on the GPU
    with pytest.raises(ValueError):
        B.make_paged_cache(torch.zeros(2, 1, 16, 64), torch.zeros(2, 1, 16, 64))
    with pytest.raises(ValueError):
        B._rows(torch.zeros(3, 2, 64))
    with pytest.raises(ValueError):
        B.make_adapters(torch.zeros(2, 8, 16), torch.zeros(2, 32, 16))


# ---- pins of the oracle -----------------------------------------------------------------------


def test_oracle_bookkeeping_keeps_every_page_in_one_place():
    rng = np.random.default_rng(0)
    for _ in range(60):
        P, B_, cols = int(rng.choice([16, 32])), int(rng.integers(1, 9)), int(rng.integers(1, 6))
        n_pages = int(rng.integers(1, B_ * cols + 3))
        free, count = [int(x) for x in rng.permutation(n_pages)], n_pages
        table, lengths = [[-1] * cols for _ in range(B_)], [0] * B_
        for _ in range(20):
            change = [int(rng.integers(-40, 60)) for _ in range(B_)]
            most = int(rng.integers(0, 200))
            before = list(lengths)
            count, lengths, granted, starts, slots, positions, owners = O.pages_assign(free, count, table, P, lengths, change, most)
            assert [b + g for b, g in zip(before, granted)] == lengths and min(lengths) >= 0
            held = [p for b in range(B_) for p in table[b] if p >= 0]
            assert sorted(held + free[:count]) == list(range(n_pages))
            for b in range(B_):
                k = -(-lengths[b] // P)
                assert all(p >= 0 for p in table[b][:k]) and all(p == -1 for p in table[b][k:])
                mine = [s for s, o in zip(slots, owners) if o == b]
                if granted[b] > 0:
                    assert mine == [table[b][r // P] * P + r % P for r in range(before[b], lengths[b])]
                else:
                    assert all(s == -1 for s in mine)
            assert len(slots) == most and starts[0] == 0 and (np.diff(starts) >= 0).all()


def test_oracle_attention_is_the_dense_librarys():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((9, 2, 16, 8)), rng.standard_normal((9, 2, 16, 8)), rng.standard_normal((3, 4, 8))
    table, lengths = [[3, 5, 1], [0, 8, 2], [7, 7, 7]], [40, 17, 0]
    out, mag = O.attention(q, k, v, table, lengths, 0.3)
    for b in range(2):
        dense = lambda x: torch.from_numpy(np.repeat(np.concatenate([x[p] for p in table[b]], 1)[:, :lengths[b]], 2, 0))
        want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[b][:, None]), dense(k), dense(v), scale=0.3)
        np.testing.assert_allclose(out[b], want[:, 0].numpy(), atol=1e-12)
    assert (out[2] == 0).all() and (mag >= np.abs(out) - 1e-12).all()


def test_oracle_adapters_are_a_change_of_the_weight():
    rng = np.random.default_rng(2)
    a, b, x = rng.standard_normal((3, 16, 24)), rng.standard_normal((3, 40, 8)), rng.standard_normal((5, 24))
    ids, scale = [2, -1, 0, 7, 2], [0.5, 1.0, 2.0]
    y, _, _ = O.adapters(x, np.zeros((5, 40)), a, b, scale, ids, [16, 40], 8)
    for m, i in enumerate(ids):
        w = np.zeros((40, 24)) if not 0 <= i < 3 else scale[i] * np.concatenate([b[i, :16] @ a[i, :8], b[i, 16:] @ a[i, 8:]])
        np.testing.assert_allclose(y[m], w @ x[m], atol=1e-12)
