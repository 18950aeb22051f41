"""The host side of serving drafted trees: the pairs' increments, cos and sin from a fixed-point angle (the library's own
source built for the host), refusals, workspace sizes, and pins of the oracle."""
import ctypes as C
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import tree_oracle as O
from paper_2604_16498_amd import binding as B
from paper_2604_16498_amd import build

SHIM = """
#define __host__
#define __device__
#include "%s"
extern "C" void turn_all(const unsigned long* p, float* c, float* s, long n) {
  for (long i = 0; i < n; ++i) forge::turn_cos_sin(p[i] >> 32, c[i], s[i]);
}
extern "C" void turned_all(const int* p, const unsigned long* inc, unsigned* top, long n) {
  for (long i = 0; i < n; ++i) top[i] = forge::turned(p[i], inc[i]);
}
"""


def test_turns_to_cos_and_sin(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    src, lib = tmp_path / "shim.cpp", tmp_path / "shim.so"
    src.write_text(SHIM % os.path.join(build.CSRC, "angles.hpp"))
    subprocess.run(["g++", "-O2", "-shared", "-fPIC", "-mfma", "-ffp-contract=off", str(src), "-o", str(lib)], check=True)
    rng = np.random.default_rng(3)
    eighths = np.arange(8, dtype=np.uint64) << np.uint64(61)
    near = np.concatenate([eighths + np.uint64(d) for d in (0, 1, 1 << 31, 1 << 32, 1 << 40)] +
                          [eighths - np.uint64(d) for d in (1, 1 << 31, 1 << 32, 1 << 40)])
    phase = np.concatenate([rng.integers(0, 2**64, 500000, dtype=np.uint64), near])
    c, s = np.empty(phase.size, np.float32), np.empty(phase.size, np.float32)
    ptr = lambda a: a.ctypes.data_as(C.c_void_p)
    C.CDLL(str(lib)).turn_all(ptr(phase), ptr(c), ptr(s), C.c_long(phase.size))
    angle = phase.astype(np.float64) * (2 * math.pi / 2.0**64)
    # the angle: half a unit of fp32 at pi/4 twice (conversion, product) and 2^-32 turns; the series: three roundings near 1
    bound = 2 * 2.0**-25 + 2 * math.pi * 2.0**-32 + 3 * 2.0**-25
    assert max(np.abs(c - np.cos(angle)).max(), np.abs(s - np.sin(angle)).max()) <= bound
    # positions of any sign: the top of the product modulo 2^64
    p = np.concatenate([rng.integers(-2**31, 2**31, 100000), [0, 1, -1, 2**31 - 1, -2**31]]).astype(np.int32)
    inc = rng.integers(0, 2**64, p.size, dtype=np.uint64)
    top = np.empty(p.size, np.uint32)
    C.CDLL(str(lib)).turned_all(ptr(p), ptr(inc), ptr(top), C.c_long(p.size))
    want = np.array([int(a) * int(b) % 2**64 >> 32 for a, b in zip(p, inc)], np.uint32)
    np.testing.assert_array_equal(top, want)


@pytest.mark.parametrize("scaling", list(B.ROPE_SCALING))
@pytest.mark.parametrize("rot", [4, 16, 64, 128, 256])
def test_increments(scaling, rot):
    for base, by, context, low, high in ((10000.0, 1.0, 100.0, 1.0, 32.0), (10000.0, 8.0, 4096.0, 1.0, 4.0),
                                         (500000.0, 2.5, 8192.0, 0.5, 32.0)):
        inc, factor = B.forge_rope_increments(base, rot, scaling, by, context, low, high)
        theta, want = O.frequencies(base, rot, scaling, by, context, low, high)
        got = inc.double().numpy() / 2.0**64 * 2 * math.pi
        assert inc.shape == (rot // 2,) and (inc >= 0).all()
        np.testing.assert_allclose(got, theta, rtol=1e-14, atol=1e-18)
        assert factor == np.float32(want)


def test_increments_refuse():
    inc, f = (C.c_uint64 * 512)(), C.c_float()
    call = lambda base=1e4, rot=64, kind=0, by=2.0, ctx=4096.0, lo=1.0, hi=4.0: B.lib().forge_rope_increments(
        base, rot, kind, by, ctx, lo, hi, inc, C.byref(f))
    assert call() == 0
    for bad in (dict(base=1.0), dict(base=math.inf), dict(base=math.nan), dict(rot=0), dict(rot=63), dict(rot=1026),
                dict(kind=5), dict(kind=-1), dict(kind=1, by=0.5), dict(kind=1, by=math.nan), dict(kind=2, rot=2),
                dict(kind=2, by=1e300, base=1e300), dict(kind=3, ctx=0.0), dict(kind=3, lo=0.0), dict(kind=3, lo=4.0),
                dict(kind=4, hi=math.inf), dict(kind=4, ctx=math.nan)):
        assert call(**bad) == 1, bad
    assert B.lib().forge_rope_increments(1e4, 64, 0, 1.0, 0.0, 0.0, 0.0, None, C.byref(f)) == 1


def _cache(**kw):
    c = B.KvCache()
    c.type, c.dt, c.n_layers, c.batch, c.kv_heads, c.cap, c.head_dim = 1, 1, 1, 2, 4, 128, 64
    c.head_stride, c.batch_stride = 128 * 64, 4 * 128 * 64
    c.k, c.v, c.k_scale, c.v_scale = 0x10000, 0x20000, 0x30000, 0x40000
    for name, v in kw.items():
        setattr(c, name, v)
    return c


def _heads(ptr=0x50000, bs=4096, ts=1024, hs=64):
    return B.Heads(ptr, bs, ts, hs)


def _rope(**kw):
    r = B.RopeDesc(64, 0, 1.0, 0x60000)
    for name, v in kw.items():
        setattr(r, name, v)
    return r


BAD_CACHES = [(dict(k=None), 1), (dict(k=0x10004), 1), (dict(v=0x10000), 1), (dict(type=3), 1), (dict(dt=2), 1), (dict(dt=0), 2),
              (dict(head_dim=96), 2), (dict(batch=0), 1), (dict(kv_heads=0), 1), (dict(cap=0), 1), (dict(n_layers=0), 1),
              (dict(k_scale=None), 1), (dict(v_scale=0x30000), 1), (dict(k_scale=0x30002), 1), (dict(head_stride=64), 1),
              (dict(head_stride=128 * 64 + 8), 1), (dict(batch_stride=4 * 128 * 64 + 32), 1), (dict(batch=70000), 2),
              (dict(kv_heads=40000), 2), (dict(n_layers=2, layer_stride=0), 1)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_a_bad_cache_is_refused_everywhere(bad, status):
    l, c, ref = B.lib(), _cache(**bad), C.byref
    x, p = _heads(), C.c_void_p(0x70000)
    assert l.forge_kv_append(ref(c), 0, None, ref(x), ref(x), None, None, 0, p, None, 1, 10, None) == status
    assert l.forge_kv_read(ref(c), 0, p, C.c_void_p(0x80000), None, 1, 10, None) == status
    assert l.forge_attn_tree(ref(c), 0, ref(x), p, None, None, 4, 1, 10, 0.1, None, 0, None) == status
    assert l.forge_kv_commit(ref(c), p, p, None, 2, 10, None) == status
    assert l.forge_attn_tree_workspace_bytes(ref(c), 4, 1, 10) == 0


def test_refusals():
    l, ref, vp = B.lib(), C.byref, C.c_void_p
    c, x, p, o = _cache(), _heads(), vp(0x70000), vp(0x80000)
    attn = lambda cache=c, layer=0, q=x, out=p, sp=None, vis=None, hq=8, n=4, mp=10, scale=0.1: l.forge_attn_tree(
        ref(cache), layer, ref(q), out, sp, vis, hq, n, mp, scale, None, 0, None)
    for kw, status in ((dict(layer=1), 1), (dict(layer=-1), 1), (dict(hq=6), 1), (dict(hq=0), 1), (dict(n=0), 1), (dict(n=65), 2),
                       (dict(mp=125), 1), (dict(mp=-1), 1), (dict(mp=2**31 - 1), 1), (dict(scale=0.0), 1),
                       (dict(scale=math.nan), 1), (dict(out=None), 1), (dict(out=vp(0x70008)), 1), (dict(out=vp(0x50000)), 1),
                       (dict(out=vp(0x10000)), 1), (dict(sp=vp(0x70002)), 1), (dict(vis=vp(0x70004)), 1),
                       (dict(q=_heads(ptr=0)), 1), (dict(q=_heads(ptr=0x50008)), 1), (dict(q=_heads(ts=1028)), 1),
                       (dict(q=_heads(hs=-64)), 1), (dict(hq=80000), 2)):
        assert attn(**kw) == status, kw
    big = _cache(cap=65536, head_stride=65536 * 64, batch_stride=4 * 65536 * 64)
    assert attn(cache=big, mp=60000) == 3                              # its ranges need a workspace
    # rotation
    rope = lambda r=_rope(), a=x, y=_heads(0x90000), pos=p, n=4, heads=4, dh=64, dt=1: l.forge_rope_apply(
        ref(r), ref(a), ref(y), pos, 2, n, heads, dh, dt, None)
    for kw, status in ((dict(r=_rope(rot_dim=0)), 1), (dict(r=_rope(rot_dim=128)), 1), (dict(r=_rope(rot_dim=24)), 2),
                       (dict(r=_rope(style=2)), 1), (dict(r=_rope(factor=math.inf)), 1), (dict(r=_rope(increments=None)), 1),
                       (dict(r=_rope(increments=0x60004)), 1), (dict(pos=None), 1), (dict(pos=vp(0x70001)), 1), (dict(n=0), 1),
                       (dict(heads=0), 1), (dict(dh=72, y=_heads(0x90000, hs=72)), 2), (dict(dh=2048, y=_heads(0x90000, bs=1 << 20, ts=1 << 16, hs=2048)), 2), (dict(dt=2), 1), (dict(n=1 << 24), 2),
                       (dict(y=_heads(0x50000, hs=128)), 1), (dict(y=_heads(0x90000, hs=32)), 1), (dict(y=_heads(0x90000, ts=0)), 1)):
        assert rope(**kw) == status, kw
    # append
    app = lambda r=None, k=x, v=x, q=None, qo=None, hq=0, sp=p, pos=None, n=4, mp=10, layer=0: l.forge_kv_append(
        ref(c), layer, r, ref(k), ref(v), q, qo, hq, sp, pos, n, mp, None)
    for kw in (dict(k=_heads(ptr=0)), dict(v=_heads(ts=4)), dict(n=0), dict(n=119), dict(mp=-1), dict(layer=3), dict(sp=vp(0x70002)),
               dict(pos=vp(0x70002)), dict(r=ref(_rope(rot_dim=128))), dict(q=ref(x), qo=None, hq=4), dict(q=ref(x), qo=ref(x), hq=0),
               dict(q=ref(x), qo=ref(_heads(hs=128)), hq=4)):
        assert app(**kw) == 1, kw
    # read, commit
    assert l.forge_kv_read(ref(c), 0, p, p, None, 1, 0, None) == 1
    assert l.forge_kv_read(ref(c), 0, vp(0x10000), o, None, 1, 0, None) == 1
    assert l.forge_kv_read(ref(c), 0, p, o, None, 129, 0, None) == 1
    assert l.forge_kv_read(ref(c), 0, p, o, None, 1, 128, None) == 1
    for args in ((None, p, None, 4, 10), (p, None, None, 4, 10), (vp(0x70002), p, None, 4, 10), (p, p, None, 4, 126), (p, p, None, 0, 10)):
        assert l.forge_kv_commit(ref(c), *args, None) == 1
    assert l.forge_kv_commit(ref(c), p, p, None, 65, 10, None) == 2
    # the layer
    d = B.BlockDesc()
    assert l.forge_decoder_block_tree(ref(d), None, ref(c), 0, p, o, None, None, None, 1, 0, p, 0, None) == 1
    assert l.forge_decoder_block_tree_workspace_bytes(ref(d), ref(c), 1, 0) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    k = torch.zeros(1, 1, 64, 64)
    with pytest.raises(ValueError):
        B.make_kv_cache(k, k.clone())                      # not on the GPU
    with pytest.raises(ValueError):
        B.make_rope_desc(torch.zeros(8, dtype=torch.int64))
    with pytest.raises(ValueError):
        B._heads(torch.zeros(1, 2, 3, 64))


@pytest.mark.parametrize("dt,dh", [(1, 64), (1, 128), (0, 64)])
def test_workspace_serves_every_shorter_cache(dt, dh):
    for batch, hkv, group, n in ((1, 8, 4, 1), (3, 12, 1, 7), (5, 8, 4, 26), (1, 1, 32, 64), (64, 8, 4, 1), (1, 2, 3, 11)):
        c = _cache(type=0, dt=dt, batch=batch, kv_heads=hkv, cap=1 << 20, head_dim=dh, head_stride=dh << 20,
                   batch_stride=hkv * dh << 20)
        prev = 0
        for pos in list(range(0, 700, 13)) + list(range(700, 20000, 571)) + [200000]:
            need = B.forge_attn_tree_workspace_bytes(c, hkv * group, n, pos)
            assert need >= prev
            prev = need


# ---- pins of the oracle -----------------------------------------------------------------------


def test_oracle_rotation_is_a_complex_product():
    rng = np.random.default_rng(0)
    x, pos = rng.standard_normal((5, 32)), rng.integers(0, 10**5, 5)
    theta, _ = O.frequencies(1e4, 16)
    for style in ("half", "interleaved"):
        y = O.rotate(x, pos, theta, style, 1.5)
        take = (lambda a: a[:, :8] + 1j * a[:, 8:16]) if style == "half" else (lambda a: a[:, 0:16:2] + 1j * a[:, 1:16:2])
        np.testing.assert_allclose(take(y), take(x) * 1.5 * np.exp(1j * pos[:, None] * theta), atol=1e-9)
        np.testing.assert_array_equal(y[:, 16:], x[:, 16:])
        np.testing.assert_allclose(O.rotate(O.rotate(x, pos, theta, style), -pos, theta, style), x, atol=1e-9)


def test_oracle_scalings():
    plain, _ = O.frequencies(1e4, 64)
    assert np.allclose(O.frequencies(1e4, 64, "linear", 4.0)[0], plain / 4)
    base = O.frequencies(1e4, 64, "base", 4.0)[0]
    assert base[0] == plain[0] and np.isclose(base[-1], plain[-1] / 4)          # the slowest pair squeezed by all of it
    for kind in ("bands", "ramp"):
        t, f = O.frequencies(1e4, 64, kind, 4.0, 4096.0, 1.0, 32.0)
        assert t[0] == plain[0] and np.isclose(t[-1], plain[-1] / 4) and (np.diff(t) < 0).all()
        assert f == (1.0 if kind == "bands" else 0.1 * math.log(4.0) + 1)


def test_oracle_e4m3_is_torchs():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    np.testing.assert_array_equal(O.e4m3_values(), codes.double().numpy())


def test_oracle_attention_is_the_masked_librarys():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((2, 3, 4, 8)), rng.standard_normal((2, 2, 9, 8)), rng.standard_normal((2, 2, 9, 8))
    pos, vis = [4, 0], [[1, 3, 5], [0, 2, 6]]
    out, mag = O.tree_attention(q, k, v, pos, vis, 0.3)
    mask = torch.zeros(2, 1, 3, 9, dtype=torch.bool)
    for b in range(2):
        for t in range(3):
            mask[b, 0, t, :pos[b]] = True
            for j in range(3):
                mask[b, 0, t, pos[b] + j] = bool(vis[b][t] >> j & 1)
    rep = lambda a: torch.from_numpy(np.repeat(a, 2, 1))
    want = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q).transpose(1, 2), rep(k), rep(v), mask, scale=0.3)
    want = torch.nan_to_num(want).transpose(1, 2).numpy()
    np.testing.assert_allclose(out, want, atol=1e-12)
    assert (out[1, 0] == 0).all() and (mag >= np.abs(out) - 1e-12).all()
