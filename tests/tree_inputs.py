"""Inputs of the drafted-tree tests: random trees, their bits, caches in every type (no arithmetic of the operators here)."""
import numpy as np
import torch

from paper_2604_16498_amd import inputs as I


def parents(rng, n):
    return [t - 1 if rng.random() < 0.5 else int(rng.integers(max(-1, t - 6), t)) for t in range(n)]


def ancestor_bits(par):
    bits = []
    for t, p in enumerate(par):
        bits.append((bits[p] if p >= 0 else 0) | 1 << t)
    return bits


def depths(par):
    d = []
    for p in par:
        d.append(d[p] + 1 if p >= 0 else 0)
    return d


def signed(bits):
    return [[b - (1 << 64) if b >> 63 else b for b in row] for row in bits]


def normal(rng, shape, bf16=True, std=1.0):
    a = (rng.standard_normal(shape) * std).astype(np.float32)
    return I.bf16_round(a) if bf16 else a


def gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def cache_arrays(rng, store, shape):
    """(tensors k, v, k_scale, v_scale on the GPU; the values they stand for, fp64): codes and scales drawn directly, every row
    another size."""
    if store in ("bf16", "fp32"):
        dt = torch.bfloat16 if store == "bf16" else torch.float32
        k, v = (normal(rng, shape, store == "bf16") for _ in range(2))
        return [gpu(k, dt), gpu(v, dt), None, None], [k.astype(np.float64), v.astype(np.float64)]
    tensors, values = [], []
    for _ in range(2):
        if store == "int8":
            codes = torch.from_numpy(rng.integers(-127, 128, shape).astype(np.int8))
            held = codes.double().numpy()
            top = 73.0
        else:
            codes = torch.from_numpy((rng.standard_normal(shape) * 100).clip(-448, 448).astype(np.float32)).to(torch.float8_e4m3fn)
            held = codes.float().numpy().astype(np.float64)
            top = 100.0
        scale = (np.exp2(rng.uniform(-2.0, 1.0, shape[:-1])) / top).astype(np.float32)
        tensors.append((codes.cuda(), gpu(scale)))
        values.append(held * scale[..., None].astype(np.float64))
    return [tensors[0][0], tensors[1][0], tensors[0][1], tensors[1][1]], values
