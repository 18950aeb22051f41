"""ctypes binding of the forge C ABI (include/forge.h).

Argument marshalling only: every function here takes torch tensors that already
live on the GPU, passes their device pointers, sizes and the current HIP stream
to the entry point of the same name, and raises :class:`ForgeError` on a
non-zero status.  No step of the computation runs in Python or in torch ops.
The shared library must exist (``python -m paper_2604_16498_amd.build``); there
is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional, Sequence

import torch

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libforge.so")

FORGE_F32, FORGE_BF16 = 0, 1
ACT = {"none": 0, "gelu_tanh": 1, "relu": 2, "silu": 3, "swiglu": 4, "gelu_erf": 5}
NORM = {"layernorm": 0, "rmsnorm": 1}
KV = {"same": 0, "int8": 1, "fp8": 2}
ROPE_STYLE = {"half": 0, "interleaved": 1}
ROPE_SCALING = {"none": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}


class ForgeError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s" % (where, status_string(status)))


class BlockDesc(C.Structure):
    _fields_ = [
        ("d_model", C.c_int), ("q_heads", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int),
        ("d_ff", C.c_int), ("norm", C.c_int), ("eps", C.c_float), ("mlp_act", C.c_int),
        ("use_rope", C.c_int), ("rope_base", C.c_float), ("dt", C.c_int),
        ("norm1_g", C.c_void_p), ("norm1_b", C.c_void_p), ("w_qkv", C.c_void_p), ("b_qkv", C.c_void_p),
        ("w_o", C.c_void_p), ("b_o", C.c_void_p), ("norm2_g", C.c_void_p), ("norm2_b", C.c_void_p),
        ("w_up", C.c_void_p), ("b_up", C.c_void_p), ("w_down", C.c_void_p), ("b_down", C.c_void_p),
        ("s_qkv", C.c_void_p), ("s_o", C.c_void_p), ("s_up", C.c_void_p), ("s_down", C.c_void_p),
    ]


class Heads(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("batch_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class RopeDesc(C.Structure):
    _fields_ = [("rot_dim", C.c_int), ("style", C.c_int), ("factor", C.c_float), ("increments", C.c_void_p)]


class KvCache(C.Structure):
    _fields_ = [
        ("type", C.c_int), ("dt", C.c_int), ("n_layers", C.c_int), ("batch", C.c_int), ("kv_heads", C.c_int),
        ("cap", C.c_int), ("head_dim", C.c_int), ("layer_stride", C.c_int64), ("batch_stride", C.c_int64),
        ("head_stride", C.c_int64), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
    ]


class PagePool(C.Structure):
    _fields_ = [("n_pages", C.c_int), ("page_rows", C.c_int), ("batch", C.c_int), ("table_cols", C.c_int),
                ("free_pages", C.c_void_p), ("free_count", C.c_void_p), ("table", C.c_void_p)]


class PagedCache(C.Structure):
    _fields_ = [
        ("type", C.c_int), ("dt", C.c_int), ("n_layers", C.c_int), ("n_pages", C.c_int), ("page_rows", C.c_int),
        ("kv_heads", C.c_int), ("head_dim", C.c_int), ("layer_stride", C.c_int64), ("page_stride", C.c_int64),
        ("head_stride", C.c_int64), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
    ]


class Adapters(C.Structure):
    _fields_ = [
        ("dt", C.c_int), ("n_adapters", C.c_int), ("rank", C.c_int), ("K", C.c_int), ("N", C.c_int), ("n_parts", C.c_int),
        ("part_end", C.c_int * 4), ("a", C.c_void_p), ("b", C.c_void_p), ("scale", C.c_void_p),
    ]


class ModelDesc(C.Structure):
    _fields_ = [
        ("n_layers", C.c_int), ("vocab", C.c_int), ("n_pos", C.c_int), ("logits_ld", C.c_int),
        ("layers", C.POINTER(BlockDesc)),
        ("wte", C.c_void_p), ("wpe", C.c_void_p), ("normf_g", C.c_void_p), ("normf_b", C.c_void_p),
    ]


_lib = None

_vp, _i, _f, _sz, _i64 = C.c_void_p, C.c_int, C.c_float, C.c_size_t, C.c_int64
_ip, _szp = C.POINTER(C.c_int), C.POINTER(C.c_size_t)
_d, _hp, _rp, _kvp = C.c_double, C.POINTER(Heads), C.POINTER(RopeDesc), C.POINTER(KvCache)
_pgp, _pcp, _adp = C.POINTER(PagePool), C.POINTER(PagedCache), C.POINTER(Adapters)

# name -> (restype, argtypes); the single list of what include/forge.h declares
SIGNATURES = {
    "forge_status_string": (C.c_char_p, [_i]),
    "forge_version": (_i, []),
    "forge_attn_fused_workspace_bytes": (_sz, [_i, _i, _i, _i, _i, _i, _i]),
    "forge_attn_fused": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i64, _i64, _f, _i, _i, _vp, _sz, _vp]),
    "forge_attn_fused_masked": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i64, _i64, _i64, _i64, _f, _i,
                                     _i, _vp]),
    "forge_gemm_workspace_bytes": (_sz, [_i, _i, _i, _i, _i]),
    "forge_gemm_variant": (C.c_char_p, [_i, _i, _i, _i, _i, _i]),
    "forge_gemm_bias_gelu": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _vp, _sz, _vp]),
    "forge_quantize_int8": (_i, [_vp, _vp, _vp, _i, _i, _i, _vp]),
    "forge_deinterleave_gated_rows": (_i, [_vp, _vp, _i, C.c_size_t, _vp]),
    "forge_gemm_w8_workspace_bytes": (_sz, [_i, _i, _i, _i]),
    "forge_gemm_w8": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _vp, _sz, _vp]),
    "forge_residual_norm": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _i, _i, _f, _i, _i, _vp]),
    "forge_rope": (_i, [_vp, _i, _i, _i, _i, _i64, _i64, _i, _i, _f, _i, _vp]),
    "forge_embed": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i, _i, _vp]),
    "forge_decoder_block_workspace_bytes": (_sz, [C.POINTER(BlockDesc), _i, _i, _i]),
    "forge_decoder_block": (_i, [C.POINTER(BlockDesc), _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _sz, _vp]),
    "forge_model_workspace_bytes": (_sz, [C.POINTER(ModelDesc), _i, _i, _i]),
    "forge_model_forward": (_i, [C.POINTER(ModelDesc), _vp, _vp, _vp, _vp, _i, _i, _i, _i, _vp, _sz, _vp]),
    "forge_attn_decode_varlen": (_i, [_vp, _vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i64, _i64, _f, _i, _vp, _sz, _vp]),
    "forge_trace_start": (_i, [_i, _vp]),
    "forge_trace_stop": (_i, [_ip, _ip, C.POINTER(C.c_float), _i]),
    "forge_attn_decode_static_max_bytes": (_sz, []),
    "forge_attn_decode_static": (_i, [_vp, _vp, _vp, _vp, _i, _i, _i, _i, _i, _i64, _i64, _f, _vp]),
    "forge_decoder_block_decode": (_i, [C.POINTER(BlockDesc), _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _vp, _sz, _vp]),
    "forge_model_decode": (_i, [C.POINTER(ModelDesc), _vp, _vp, _vp, _vp, _vp, _i, _i, _i, _vp, _sz, _vp]),
    "forge_compiled_bind_decode": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "forge_rope_increments": (_i, [_d, _i, _i, _d, _d, _d, _d, C.POINTER(C.c_uint64), C.POINTER(_f)]),
    "forge_rope_apply": (_i, [_rp, _hp, _hp, _vp, _i, _i, _i, _i, _i, _vp]),
    "forge_kv_append": (_i, [_kvp, _i, _rp, _hp, _hp, _hp, _hp, _i, _vp, _vp, _i, _i, _vp]),
    "forge_kv_read": (_i, [_kvp, _i, _vp, _vp, _vp, _i, _i, _vp]),
    "forge_attn_tree_workspace_bytes": (_sz, [_kvp, _i, _i, _i]),
    "forge_attn_tree": (_i, [_kvp, _i, _hp, _vp, _vp, _vp, _i, _i, _i, _f, _vp, _sz, _vp]),
    "forge_kv_commit": (_i, [_kvp, _vp, _vp, _vp, _i, _i, _vp]),
    "forge_decoder_block_tree_workspace_bytes": (_sz, [C.POINTER(BlockDesc), _kvp, _i, _i]),
    "forge_decoder_block_tree": (_i, [C.POINTER(BlockDesc), _rp, _kvp, _i, _vp, _vp, _vp, _vp, _vp, _i, _i, _vp, _sz, _vp]),
    "forge_pages_assign": (_i, [_pgp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i, _vp]),
    "forge_paged_append": (_i, [_pcp, _i, _rp, _hp, _hp, _hp, _hp, _i, _vp, _vp, _i, _vp]),
    "forge_paged_read": (_i, [_pcp, _i, _hp, _hp, _vp, _i, _vp]),
    "forge_attn_paged_workspace_bytes": (_sz, [_pcp, _i, _i, _i]),
    "forge_attn_paged": (_i, [_pcp, _i, _hp, _vp, _vp, _vp, _i, _i, _i, _i, _f, _vp, _sz, _vp]),
    "forge_adapters_workspace_bytes": (_sz, [_adp, _i]),
    "forge_adapters_add": (_i, [_adp, _vp, _vp, _vp, _vp, _i, _i, _vp, _sz, _vp]),
    "forge_plan_liveness": (_i, [_i, _ip, _ip, _ip, _i, _ip, _ip]),
    "forge_plan_dead_after": (_i, [_i, _ip, _i, _ip, _ip]),
    "forge_plan_linear_scan": (_i, [_i, _ip, _ip, _ip, _ip]),
    "forge_plan_workspace": (_i, [_i, _ip, _ip, _szp, _szp, _szp, _ip]),
    "forge_compile_model": (_i, [C.POINTER(ModelDesc), _i, _i, _i, _i, C.POINTER(_vp)]),
    "forge_compiled_destroy": (None, [_vp]),
    "forge_compiled_workspace_bytes": (_sz, [_vp]),
    "forge_compiled_counts": (_i, [_vp, _ip, _ip, _ip, _ip]),
    "forge_compiled_program": (_i, [_vp, _ip, _ip, _ip, _ip, _szp, _szp]),
    "forge_compiled_bind": (_i, [_vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "forge_compiled_run": (_i, [_vp, _vp]),
}


def lib() -> C.CDLL:
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError("%s is missing: build it with `python -m paper_2604_16498_amd.build`"
                              % _LIB_PATH)
        l = C.CDLL(_LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


def status_string(status: int) -> str:
    return lib().forge_status_string(status).decode()


def _p(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("forge tensors must be contiguous GPU tensors")
    return t.data_ptr()


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return FORGE_F32
    if t.dtype == torch.bfloat16:
        return FORGE_BF16
    raise ValueError("unsupported dtype %s" % t.dtype)


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(d: Optional[int] = None):
    """The current stream of the current device, which is d where the caller has asked for it already."""
    if _raw_stream is None:
        return C.c_void_p(torch.cuda.current_stream().cuda_stream)
    # the same handle without the Stream object around it (2.8 -> 0.2 us a call)
    return _raw_stream(_device() if d is None else d)


def _ws(t: Optional[torch.Tensor]):
    return (None, 0) if t is None else (_p(t), t.nbytes)


def _check(status: int, where: str):
    if status != 0:
        raise ForgeError(status, where)


def workspace(nbytes: int, device="cuda") -> Optional[torch.Tensor]:
    """Device scratch of at least nbytes (None when nothing is needed)."""
    return None if nbytes == 0 else torch.empty(nbytes, dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------------------------


def forge_attn_fused_workspace_bytes(batch, q_heads, kv_heads, q_len, kv_len, head_dim, dtype) -> int:
    dt = FORGE_BF16 if dtype == torch.bfloat16 else FORGE_F32
    return lib().forge_attn_fused_workspace_bytes(batch, q_heads, kv_heads, q_len, kv_len, head_dim, dt)


def forge_attn_fused(q, k, v, out, kv_len=None, scale=None, causal=True, workspace=None,
                     kv_batch_stride=None, kv_head_stride=None):
    """q [B,Hq,Sq,dh]; k, v [B,Hkv,cap,dh] (cap >= kv_len); out [B,Sq,Hq*dh]."""
    B, Hq, Sq, dh = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    kv_len = cap if kv_len is None else kv_len
    scale = dh ** -0.5 if scale is None else scale
    hs = cap * dh if kv_head_stride is None else kv_head_stride
    bs = Hkv * hs if kv_batch_stride is None else kv_batch_stride
    wp, wb = _ws(workspace)
    _check(lib().forge_attn_fused(_p(q), _p(k), _p(v), _p(out), B, Hq, Hkv, Sq, kv_len, dh, bs, hs,
                                  scale, int(causal), _dt(q), wp, wb, _stream()), "forge_attn_fused")
    return out


def forge_attn_fused_masked(q, k, v, mask, out, kv_len=None, scale=None, causal=False):
    """As forge_attn_fused, with an additive fp32 mask [B or 1, Hq or 1, Sq, kv_len] on the
    scaled scores (size-1 axes broadcast)."""
    B, Hq, Sq, dh = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    kv_len = cap if kv_len is None else kv_len
    scale = dh ** -0.5 if scale is None else scale
    hs = cap * dh
    bs = Hkv * hs
    assert mask.dtype == torch.float32 and mask.is_contiguous() and mask.shape[2:] == (Sq, kv_len)
    mhs = 0 if mask.shape[1] == 1 else Sq * kv_len
    mbs = 0 if mask.shape[0] == 1 else mask.shape[1] * Sq * kv_len
    _check(lib().forge_attn_fused_masked(_p(q), _p(k), _p(v), _p(mask), _p(out), B, Hq, Hkv, Sq, kv_len, dh,
                                         bs, hs, mbs, mhs, scale, int(causal), _dt(q), _stream()),
           "forge_attn_fused_masked")
    return out


def forge_gemm_workspace_bytes(M, N, K, act, dtype) -> int:
    dt = FORGE_BF16 if dtype == torch.bfloat16 else FORGE_F32
    return lib().forge_gemm_workspace_bytes(M, N, K, ACT[act], dt)


def forge_gemm_variant(M, N, K, act, dtype, ldy=0) -> str:
    dt = FORGE_BF16 if dtype == torch.bfloat16 else FORGE_F32
    return lib().forge_gemm_variant(M, N, K, ldy, ACT[act], dt).decode()


def forge_gemm_bias_gelu(x, w, bias, residual, y, act="gelu_tanh", workspace=None, n=None):
    """y[M,:N] = act(x[M,K] w[N,K]^T + bias) (+ residual); swiglu: w is [2N,K].
    y (and residual) may be wider than N (row stride y.shape[1]); pass n=N then."""
    M, K = x.shape
    ldy = y.shape[1]
    N = ldy if n is None else n
    wp, wb = _ws(workspace)
    _check(lib().forge_gemm_bias_gelu(_p(x), _p(w), _p(bias), _p(residual), _p(y), M, N, K, ldy,
                                      ACT[act], _dt(x), wp, wb, _stream()), "forge_gemm_bias_gelu")
    return y


def forge_deinterleave_gated_rows(src):
    """src [2N, ...] with alternating gate / up rows -> new tensor, gate rows first."""
    assert src.is_cuda and src.is_contiguous() and src.shape[0] % 2 == 0
    dst = torch.empty_like(src)
    row_bytes = src[0].numel() * src.element_size()
    _check(lib().forge_deinterleave_gated_rows(_p(src), _p(dst), src.shape[0] // 2, row_bytes, _stream()),
           "forge_deinterleave_gated_rows")
    return dst


def forge_quantize_int8(w):
    """w [N,K] (bf16 or fp32, GPU) -> (q int8 [N,K], scale fp32 [N])."""
    N, K = w.shape
    q = torch.empty(N, K, dtype=torch.int8, device=w.device)
    scale = torch.empty(N, dtype=torch.float32, device=w.device)
    _check(lib().forge_quantize_int8(_p(w), _p(q), _p(scale), N, K, _dt(w), _stream()), "forge_quantize_int8")
    return q, scale


def forge_gemm_w8_workspace_bytes(M, N, K, act) -> int:
    return lib().forge_gemm_w8_workspace_bytes(M, N, K, ACT[act])


def forge_gemm_w8(x, wq, wscale, bias, residual, y, act="none", workspace=None, n=None):
    """y[M,:N] = act(x[M,K] (wq * wscale[:,None])^T + bias) (+ residual); x, y bf16, wq int8."""
    M, K = x.shape
    ldy = y.shape[1]
    N = ldy if n is None else n
    wp, wb = _ws(workspace)
    _check(lib().forge_gemm_w8(_p(x), _p(wq), _p(wscale), _p(bias), _p(residual), _p(y), M, N, K, ldy,
                               ACT[act], wp, wb, _stream()), "forge_gemm_w8")
    return y


def forge_residual_norm(x, delta, gamma, beta, h_out, y, eps=1e-5, kind="layernorm"):
    rows, d = x.shape[0] if x.dim() == 2 else x.numel() // x.shape[-1], x.shape[-1]
    _check(lib().forge_residual_norm(_p(x), _p(delta), _p(gamma), _p(beta), _p(h_out), _p(y), rows, d,
                                     eps, NORM[kind], _dt(x), _stream()), "forge_residual_norm")
    return h_out, y


def forge_rope(x, n_rows=None, row0=0, pos0=0, base=10000.0):
    """In place on x [B,H,rows_cap,dh]; rotates rows row0..row0+n_rows-1 at positions pos0.."""
    B, H, cap, dh = x.shape
    n_rows = cap - row0 if n_rows is None else n_rows
    _check(lib().forge_rope(_p(x), B, H, n_rows, dh, H * cap * dh, cap * dh, row0, pos0, base, _dt(x),
                            _stream()), "forge_rope")
    return x


def forge_embed(ids, wte, wpe, h, pos0=0):
    B, S = ids.shape
    _check(lib().forge_embed(_p(ids), _p(wte), _p(wpe), _p(h), B, S, wte.shape[1], wte.shape[0],
                             wpe.shape[0], pos0, _dt(wte), _stream()), "forge_embed")
    return h


def make_block_desc(shape, w: Dict[str, Optional[torch.Tensor]]) -> BlockDesc:
    """shape: object with the BlockShape attributes; w: name -> GPU tensor (or None).
    The returned struct holds raw pointers: keep ``w`` alive while it is in use."""
    d = BlockDesc()
    d.d_model, d.q_heads, d.kv_heads, d.head_dim, d.d_ff = (shape.d_model, shape.q_heads,
                                                            shape.kv_heads, shape.head_dim, shape.d_ff)
    d.norm = NORM[shape.norm]
    d.eps = shape.eps
    d.mlp_act = ACT[shape.mlp_act]
    d.use_rope = int(shape.use_rope)
    d.rope_base = shape.rope_base
    # int8 weights (with "s_*" scale vectors in w): the activation dtype is that of the norm gain
    d.dt = _dt(w["norm1_g"] if w.get("s_qkv") is not None else w["w_qkv"])
    for name in ("norm1_g", "norm1_b", "w_qkv", "b_qkv", "w_o", "b_o", "norm2_g", "norm2_b",
                 "w_up", "b_up", "w_down", "b_down", "s_qkv", "s_o", "s_up", "s_down"):
        t = w.get(name)
        if t is not None and (not t.is_cuda or not t.is_contiguous()):
            raise ValueError("weight %s must be a contiguous GPU tensor" % name)
        setattr(d, name, None if t is None else t.data_ptr())
    return d


def forge_decoder_block_workspace_bytes(desc: BlockDesc, batch, q_len, kv_cap) -> int:
    return lib().forge_decoder_block_workspace_bytes(C.byref(desc), batch, q_len, kv_cap)


def forge_decoder_block(desc: BlockDesc, x_in, x_out, k_cache, v_cache, pos0, workspace):
    """x_in/x_out [B,q_len,d]; caches [B,Hkv,kv_cap,dh]."""
    B, q_len, _ = x_in.shape
    kv_cap = k_cache.shape[2]
    wp, wb = _ws(workspace)
    _check(lib().forge_decoder_block(C.byref(desc), _p(x_in), _p(x_out), _p(k_cache), _p(v_cache), B,
                                     q_len, pos0, kv_cap, wp, wb, _stream()), "forge_decoder_block")
    return x_out


def make_model_desc(layer_descs: Sequence[BlockDesc], mw: Dict[str, Optional[torch.Tensor]],
                    logits_ld: int = 0) -> ModelDesc:
    """mw: wte, wpe (both or neither), normf_g, normf_b.  Keeps the layer array alive on the struct."""
    m = ModelDesc()
    arr = (BlockDesc * len(layer_descs))(*layer_descs)
    m._layer_array = arr            # owner
    m.n_layers = len(layer_descs)
    m.layers = C.cast(arr, C.POINTER(BlockDesc))
    wte, wpe = mw.get("wte"), mw.get("wpe")
    m.vocab = 0 if wte is None else wte.shape[0]
    m.n_pos = 0 if wpe is None else wpe.shape[0]
    m.logits_ld = logits_ld
    for name in ("wte", "wpe", "normf_g", "normf_b"):
        t = mw.get(name)
        setattr(m, name, None if t is None else t.data_ptr())
    return m


def forge_model_workspace_bytes(model: ModelDesc, batch, q_len, kv_cap) -> int:
    return lib().forge_model_workspace_bytes(C.byref(model), batch, q_len, kv_cap)


def forge_model_forward(model: ModelDesc, inp, out, k_cache, v_cache, pos0, workspace):
    """inp: int32 ids [B,q_len] (token model) or hidden state [B,q_len,d]; caches [L,B,Hkv,cap,dh]."""
    B, q_len = inp.shape[0], inp.shape[1]
    kv_cap = k_cache.shape[3]
    wp, wb = _ws(workspace)
    _check(lib().forge_model_forward(C.byref(model), _p(inp), _p(out), _p(k_cache), _p(v_cache), B,
                                     q_len, pos0, kv_cap, wp, wb, _stream()), "forge_model_forward")
    return out


# ---------------------------------------------------------------------------------------------
# Decode step with per-sequence positions (seq_pos: int32 GPU tensor [B]).


def forge_attn_decode_varlen(q, k, v, out, seq_pos, max_pos, scale=None, workspace=None):
    """q [B,Hq,1,dh]; k, v [B,Hkv,cap,dh]; out [B,1,Hq*dh]; sequence b attends rows [0, seq_pos[b]]."""
    B, Hq, _, dh = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    scale = dh ** -0.5 if scale is None else scale
    wp, wb = _ws(workspace)
    assert seq_pos.dtype == torch.int32 and seq_pos.numel() == B
    _check(lib().forge_attn_decode_varlen(_p(q), _p(k), _p(v), _p(out), _p(seq_pos), B, Hq, Hkv, max_pos, dh,
                                          Hkv * cap * dh, cap * dh, scale, _dt(q), wp, wb, _stream()),
           "forge_attn_decode_varlen")
    return out


OP_NAMES = ["embed", "norm", "gemm_qkv", "rope_q", "rope_k", "attn", "gemm_res", "gemm_act", "gemm"]


def forge_trace_start(capacity: int):
    _check(lib().forge_trace_start(capacity, _stream()), "forge_trace_start")


def forge_trace_stop(capacity: int):
    """-> [(operator name, milliseconds)] of the launch lists run since forge_trace_start."""
    n = C.c_int(0)
    ops = (C.c_int * capacity)()
    ms = (C.c_float * capacity)()
    _check(lib().forge_trace_stop(C.byref(n), ops, ms, capacity), "forge_trace_stop")
    return [(OP_NAMES[ops[i]], float(ms[i])) for i in range(min(n.value, capacity))]


def forge_attn_decode_static_max_bytes() -> int:
    return int(lib().forge_attn_decode_static_max_bytes())


def forge_attn_decode_static(q, k, v, out, kv_len=None, scale=None):
    """forge_attn_fused for q_len 1 (bf16, causal) with the library's own fixed scratch: no workspace.
    q [B,Hq,1,dh]; k, v [B,Hkv,cap,dh]; out [B,1,Hq*dh]."""
    B, Hq, Sq, dh = q.shape
    assert Sq == 1 and q.dtype == torch.bfloat16
    Hkv, cap = k.shape[1], k.shape[2]
    kv_len = cap if kv_len is None else kv_len
    scale = dh ** -0.5 if scale is None else scale
    _check(lib().forge_attn_decode_static(_p(q), _p(k), _p(v), _p(out), B, Hq, Hkv, kv_len, dh,
                                          Hkv * cap * dh, cap * dh, scale, _stream()),
           "forge_attn_decode_static")
    return out


def forge_decoder_block_decode(desc: BlockDesc, x_in, x_out, k_cache, v_cache, seq_pos, max_pos, workspace):
    B = x_in.shape[0]
    kv_cap = k_cache.shape[2]
    wp, wb = _ws(workspace)
    assert seq_pos.dtype == torch.int32 and seq_pos.numel() == B
    _check(lib().forge_decoder_block_decode(C.byref(desc), _p(x_in), _p(x_out), _p(k_cache), _p(v_cache),
                                            _p(seq_pos), B, max_pos, kv_cap, wp, wb, _stream()),
           "forge_decoder_block_decode")
    return x_out


def forge_model_decode(model: ModelDesc, inp, out, k_cache, v_cache, seq_pos, max_pos, workspace):
    B = inp.shape[0]
    kv_cap = k_cache.shape[3]
    wp, wb = _ws(workspace)
    assert seq_pos.dtype == torch.int32 and seq_pos.numel() == B
    _check(lib().forge_model_decode(C.byref(model), _p(inp), _p(out), _p(k_cache), _p(v_cache), _p(seq_pos), B,
                                    max_pos, kv_cap, wp, wb, _stream()), "forge_model_decode")
    return out


# ---------------------------------------------------------------------------------------------
# Drafted trees over a (quantised) cache.


def _heads(t: torch.Tensor) -> Heads:
    """A [batch, token, head, head_dim] view, any strides, head_dim dense."""
    sb, st, sh, sd = t.stride()
    if not t.is_cuda or (sd != 1 and t.shape[3] != 1):
        raise ValueError("forge needs [batch, token, head, head_dim] GPU tensors with a dense last axis")
    return Heads(t.data_ptr(), sb, st, sh)


_INT32 = torch.int32


def _int32(t: Optional[torch.Tensor], shape, what: str):
    if t is None:
        return None
    if t.dtype is not _INT32 or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous int32 GPU tensor of shape %s" % (what, tuple(shape)))
    return t.data_ptr()


def forge_rope_increments(base, rot_dim, scaling="none", by=1.0, context=0.0, low=1.0, high=4.0):
    """-> (int64 CPU tensor [rot_dim / 2] of the pairs' turns a position in units of 2^-64, factor of cos and sin)."""
    inc, factor = (C.c_uint64 * max(1, rot_dim // 2))(), C.c_float(0.0)
    _check(lib().forge_rope_increments(base, rot_dim, ROPE_SCALING[scaling], by, context, low, high, inc, C.byref(factor)),
           "forge_rope_increments")
    return torch.tensor([v - (1 << 64) if v >> 63 else v for v in inc], dtype=torch.int64), factor.value


def make_rope_desc(increments: torch.Tensor, style="half", factor=1.0) -> RopeDesc:
    """increments: int64 GPU tensor [rot_dim / 2], kept alive on the struct."""
    if increments.dtype != torch.int64 or not increments.is_cuda or not increments.is_contiguous():
        raise ValueError("increments must be a contiguous int64 GPU tensor")
    r = RopeDesc(2 * increments.numel(), ROPE_STYLE[style], factor, increments.data_ptr())
    r._increments, r._gpu = increments, increments.get_device()
    return r


def forge_rope_apply(rope: RopeDesc, x, y, positions):
    """y = rotated x; [B,n,H,dh] views (y may be x); positions int32 [B,n], any sign."""
    B, n, H, dh = x.shape
    if y.shape != x.shape or y.dtype != x.dtype:
        raise ValueError("x and y must agree in shape and dtype")
    _check(lib().forge_rope_apply(C.byref(rope), C.byref(_heads(x)), C.byref(_heads(y)), _int32(positions, (B, n), "positions"),
                                  B, n, H, dh, _dt(x), _stream()), "forge_rope_apply")
    return y


def make_kv_cache(k, v, k_scale=None, v_scale=None) -> KvCache:
    """k, v: [B,Hkv,cap,dh] or, of all layers, [L,B,Hkv,cap,dh] views whose rows are dense, in bf16, fp32, int8 or
    float8_e4m3fn; the 8-bit ones with fp32 scales of the same shape and strides without dh.  The struct keeps them alive."""
    tensors = [t for t in (k, v, k_scale, v_scale) if t is not None]
    if k.dim() not in (4, 5) or v.shape != k.shape or v.stride() != k.stride() or v.dtype != k.dtype:
        raise ValueError("k and v must be [B,Hkv,cap,dh] or [L,B,Hkv,cap,dh] tensors alike in shape, strides and dtype")
    dh = k.shape[-1]
    if any(not t.is_cuda for t in tensors) or k.stride(-1) != 1 or k.stride(-2) != dh:
        raise ValueError("a cache holds dense rows one behind another, on the GPU")
    c = KvCache()
    c.type = KV[{torch.int8: "int8", torch.float8_e4m3fn: "fp8"}.get(k.dtype, "same")]
    c.dt = FORGE_BF16 if c.type else _dt(k)
    if (c.type != 0) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
        raise ValueError("8-bit caches, and they alone, have scales")
    for s in (k_scale, v_scale):
        if s is not None and (s.dtype != torch.float32 or s.shape != k.shape[:-1] or
                              any(n > 1 and st * dh != t for n, st, t in zip(s.shape, s.stride(), k.stride()))):
            raise ValueError("scales are fp32, shaped and strided as the rows they belong to")
    (c.n_layers, sl), shape, stride = ((k.shape[0], k.stride(0)) if k.dim() == 5 else (1, 0)), k.shape[-4:], k.stride()[-4:]
    c.batch, c.kv_heads, c.cap, c.head_dim = shape
    c.layer_stride, c.batch_stride, c.head_stride = sl, stride[0], stride[1]
    c.k, c.v = k.data_ptr(), v.data_ptr()
    c.k_scale, c.v_scale = (None, None) if k_scale is None else (k_scale.data_ptr(), v_scale.data_ptr())
    c._tensors = tensors
    return c


def _cache_dt(cache: KvCache, *tensors):
    want = torch.float32 if cache.dt == FORGE_F32 else torch.bfloat16
    for t in tensors:
        if t.dtype != want:
            raise ValueError("this cache takes and gives rows in %s" % want)


def forge_kv_append(cache: KvCache, k, v, seq_pos, max_pos, rope=None, positions=None, q=None, q_out=None, layer=0):
    """k, v [B,n,Hkv,dh] views into cache rows seq_pos[b].., k rotated; q [B,n,Hq,dh] rotated into q_out (may be q)."""
    shape = k.shape
    B, n, heads, dh = shape
    if B != cache.batch or heads != cache.kv_heads or dh != cache.head_dim or v.shape != shape:
        raise ValueError("k and v must be [%d, n, %d, %d]" % (cache.batch, cache.kv_heads, cache.head_dim))
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    if q is None:
        q_heads, qp, qop = 0, None, None
        _cache_dt(cache, k, v)
    else:
        q_heads = q.shape[2]
        if q.shape != (B, n, q_heads, dh) or q_out.shape != q.shape:
            raise ValueError("q and q_out must be [%d, %d, Hq, %d]" % (B, n, dh))
        _cache_dt(cache, k, v, q, q_out)
        qp, qop = C.byref(_heads(q)), C.byref(_heads(q_out))
    _check(lib().forge_kv_append(C.byref(cache), layer, None if rope is None else C.byref(rope), C.byref(_heads(k)),
                                 C.byref(_heads(v)), qp, qop, q_heads, _int32(seq_pos, (B,), "seq_pos"),
                                 _int32(positions, (B, n), "positions"), n, max_pos, _stream()), "forge_kv_append")


def forge_kv_read(cache: KvCache, k_out, v_out, seq_pos=None, max_pos=0, layer=0):
    """k_out, v_out [B,Hkv,n,dh]: rows seq_pos[b].. (seq_pos None: max_pos..) as values in the cache's activation type."""
    B, H, n, dh = k_out.shape
    if (B, H, dh) != (cache.batch, cache.kv_heads, cache.head_dim) or v_out.shape != k_out.shape:
        raise ValueError("k_out and v_out must be [%d, %d, n, %d]" % (cache.batch, cache.kv_heads, cache.head_dim))
    _cache_dt(cache, k_out, v_out)
    _check(lib().forge_kv_read(C.byref(cache), layer, _p(k_out), _p(v_out), _int32(seq_pos, (B,), "seq_pos"), n, max_pos,
                               _stream()), "forge_kv_read")
    return k_out, v_out


def forge_attn_tree_workspace_bytes(cache: KvCache, q_heads, n, max_pos) -> int:
    return lib().forge_attn_tree_workspace_bytes(C.byref(cache), q_heads, n, max_pos)


def _visible(t: Optional[torch.Tensor], shape):
    if t is None:
        return None
    if t.dtype != torch.int64 or t.shape != shape or not t.is_cuda or not t.is_contiguous():
        raise ValueError("visible must be a contiguous int64 GPU tensor of shape %s" % (tuple(shape),))
    return t.data_ptr()


def forge_attn_tree(cache: KvCache, q, out, seq_pos, max_pos, visible=None, scale=None, workspace=None, layer=0):
    """q [B,n,Hq,dh] view; out [B,n,Hq*dh]; visible int64 [B,n]: bit i of entry t: new token t sees new row i (None: causal)."""
    B, n, H, dh = q.shape
    if B != cache.batch or dh != cache.head_dim or out.shape != (B, n, H * dh):
        raise ValueError("q must be [%d, n, Hq, %d] and out [%d, n, Hq * %d]" % (cache.batch, cache.head_dim, cache.batch, cache.head_dim))
    _cache_dt(cache, q, out)
    wp, wb = _ws(workspace)
    _check(lib().forge_attn_tree(C.byref(cache), layer, C.byref(_heads(q)), _p(out), _int32(seq_pos, (B,), "seq_pos"),
                                 _visible(visible, (B, n)), H, n, max_pos, dh ** -0.5 if scale is None else scale, wp, wb,
                                 _stream()), "forge_attn_tree")
    return out


def forge_kv_commit(cache: KvCache, path, accepted, seq_pos, max_pos):
    """Row seq_pos[b] + j of every layer takes row seq_pos[b] + path[b, j], j < accepted[b]; path int32 [B,n], rising."""
    B, n = path.shape
    if B != cache.batch or accepted is None:
        raise ValueError("path must be [%d, n], accepted [%d]" % (cache.batch, cache.batch))
    _check(lib().forge_kv_commit(C.byref(cache), _int32(path, (B, n), "path"), _int32(accepted, (B,), "accepted"),
                                 _int32(seq_pos, (B,), "seq_pos"), n, max_pos, _stream()), "forge_kv_commit")


def forge_decoder_block_tree_workspace_bytes(desc: BlockDesc, cache: KvCache, n, max_pos) -> int:
    return lib().forge_decoder_block_tree_workspace_bytes(C.byref(desc), C.byref(cache), n, max_pos)


def forge_decoder_block_tree(desc: BlockDesc, cache: KvCache, x_in, x_out, seq_pos, max_pos, workspace, rope=None,
                             positions=None, visible=None, layer=0):
    """x_in / x_out [B,n,d]: one decoder layer over n new tokens per sequence, rows in `cache`."""
    B, n, _ = x_in.shape
    if B != cache.batch or x_out.shape != x_in.shape or x_in.shape[2] != desc.d_model:
        raise ValueError("x_in and x_out must be [%d, n, %d]" % (cache.batch, desc.d_model))
    _cache_dt(cache, x_in, x_out)
    wp, wb = _ws(workspace)
    _check(lib().forge_decoder_block_tree(C.byref(desc), None if rope is None else C.byref(rope), C.byref(cache), layer, _p(x_in),
                                          _p(x_out), _int32(seq_pos, (B,), "seq_pos"), _int32(positions, (B, n), "positions"),
                                          _visible(visible, (B, n)), n, max_pos, wp, wb, _stream()),
           "forge_decoder_block_tree")
    return x_out


# ---------------------------------------------------------------------------------------------
# Many requests over one pool of cache pages.


def make_page_pool(free_pages, free_count, table, page_rows) -> PagePool:
    """free_pages int32 [n_pages], the stack of free pages' numbers, of which free_count [1] count; table int32 [batch, cols].
    The struct keeps them alive."""
    if free_pages.dim() != 1 or table.dim() != 2:
        raise ValueError("free_pages must be [n_pages], table [batch, cols]")
    p = PagePool(free_pages.shape[0], page_rows, table.shape[0], table.shape[1], _int32(free_pages, free_pages.shape, "free_pages"),
                 _int32(free_count, (1,), "free_count"), _int32(table, table.shape, "table"))
    return _keeping(p, (free_pages, free_count, table))


def _keeping(desc, tensors):
    """A descriptor keeps its tensors alive, and the GPU that they lie on."""
    desc._tensors, desc._gpu = tensors, tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != desc._gpu:
            raise ValueError("a descriptor's tensors are on GPU %d and GPU %d" % (desc._gpu, t.get_device()))
    return desc


# The work goes to the current device's (d) stream: a call's tensors have to lie there, and its descriptors' (one filled in by hand does not
# say where).  A device that is not d is a tensor on the CPU, too (-1), so that this one question is the only one.


def _refuse(gpu: int, d: int, otherwise: str):
    raise ValueError("a tensor of the call is on GPU %d, the current one is %d" % (gpu, d) if gpu not in (d, -1) else otherwise)


def _here(desc, d: int):
    gpu = getattr(desc, "_gpu", d)
    if gpu != d:
        _refuse(gpu, d, "a descriptor of tensors on the CPU")


def _vector(t: torch.Tensor, n: int, what: str, d: int):
    if t.get_device() != d or t.dtype is not _INT32 or t.numel() != n or not t.is_contiguous():
        _refuse(t.get_device(), d, "%s must be a contiguous int32 GPU tensor of %d entries" % (what, n))
    return t.data_ptr()


def _at(t: torch.Tensor, d: int):
    if t.get_device() != d or not t.is_contiguous():
        _refuse(t.get_device(), d, "forge tensors must be contiguous GPU tensors")
    return t.data_ptr()


def _ws_at(t: Optional[torch.Tensor], d: int):
    return (None, 0) if t is None else (_at(t, d), t.nbytes)


def forge_pages_assign(pool: PagePool, lengths, change, lengths_out, granted, starts, slots=None, positions=None, owners=None):
    """Lengths change by change[b] (int32 [batch]), pages move, and every new token gets slots, positions and owners (int32
    [max_tokens], or all None); granted [batch]: the changes that took place; starts [batch + 1]: the tokens of every request."""
    B, d = pool.batch, _device()
    _here(pool, d)
    if slots is None:
        if positions is not None or owners is not None:
            raise ValueError("slots, positions and owners come together")
        T, sp, pp, op = 0, None, None, None
    else:
        T = slots.numel()
        sp, pp, op = _vector(slots, T, "slots", d), _vector(positions, T, "positions", d), _vector(owners, T, "owners", d)
    _check(lib().forge_pages_assign(C.byref(pool), _vector(lengths, B, "lengths", d), _vector(change, B, "change", d),
                                    _vector(lengths_out, B, "lengths_out", d), _vector(granted, B, "granted", d),
                                    _vector(starts, B + 1, "starts", d), sp, pp, op, T, _stream(d)), "forge_pages_assign")


def make_paged_cache(k, v, k_scale=None, v_scale=None) -> PagedCache:
    """k, v: [pages,Hkv,rows,dh] or, of all layers, [L,pages,Hkv,rows,dh] views whose rows are dense, in bf16, fp32, int8 or
    float8_e4m3fn; the 8-bit ones with fp32 scales of the same shape and strides without dh.  The struct keeps them alive."""
    flat = make_kv_cache(k, v, k_scale, v_scale)          # (the same views: pages in the place of sequences)
    return _keeping(PagedCache(flat.type, flat.dt, flat.n_layers, flat.batch, flat.cap, flat.kv_heads, flat.head_dim, flat.layer_stride,
                               flat.batch_stride, flat.head_stride, flat.k, flat.v, flat.k_scale, flat.v_scale), flat._tensors)


def _rows(t: torch.Tensor, d: Optional[int] = None) -> Heads:
    """A [token, head, head_dim] view on GPU d, any strides, head_dim dense."""
    st, sh, sd = t.stride()
    if t.get_device() != d or (sd != 1 and t.shape[2] != 1):
        _refuse(t.get_device(), d, "forge needs [token, head, head_dim] GPU tensors with a dense last axis")
    return Heads(t.data_ptr(), 0, st, sh)


def forge_paged_append(cache: PagedCache, k, v, slots, rope=None, positions=None, q=None, q_out=None, layer=0):
    """k, v [T,Hkv,dh] views into the rows of slots [T], k rotated at positions [T]; q [T,Hq,dh] rotated into q_out (may be q)."""
    (T, heads, dh), d = k.shape, _device()
    _here(cache, d)
    if rope is not None:
        _here(rope, d)
    if heads != cache.kv_heads or dh != cache.head_dim or v.shape != k.shape:
        raise ValueError("k and v must be [T, %d, %d]" % (cache.kv_heads, cache.head_dim))
    if (q is None) != (q_out is None) or slots is None:
        raise ValueError("q and q_out come together, slots always")
    if q is None:
        q_heads, qp, qop = 0, None, None
        _cache_dt(cache, k, v)
    else:
        q_heads = q.shape[1]
        if q.shape != (T, q_heads, dh) or q_out.shape != q.shape:
            raise ValueError("q and q_out must be [%d, Hq, %d]" % (T, dh))
        _cache_dt(cache, k, v, q, q_out)
        qp, qop = C.byref(_rows(q, d)), C.byref(_rows(q_out, d))
    _check(lib().forge_paged_append(C.byref(cache), layer, None if rope is None else C.byref(rope), C.byref(_rows(k, d)), C.byref(_rows(v, d)),
                                    qp, qop, q_heads, _vector(slots, T, "slots", d),
                                    None if positions is None else _vector(positions, T, "positions", d), T, _stream(d)), "forge_paged_append")


def forge_paged_read(cache: PagedCache, k_out, v_out, slots, layer=0):
    """k_out, v_out [T,Hkv,dh] views: the rows of slots [T] as values in the cache's activation type."""
    (T, heads, dh), d = k_out.shape, _device()
    _here(cache, d)
    if (heads, dh) != (cache.kv_heads, cache.head_dim) or v_out.shape != k_out.shape or slots is None:
        raise ValueError("k_out and v_out must be [T, %d, %d]" % (cache.kv_heads, cache.head_dim))
    _cache_dt(cache, k_out, v_out)
    _check(lib().forge_paged_read(C.byref(cache), layer, C.byref(_rows(k_out, d)), C.byref(_rows(v_out, d)),
                                  _vector(slots, T, "slots", d), T, _stream(d)), "forge_paged_read")
    return k_out, v_out


def forge_attn_paged_workspace_bytes(cache: PagedCache, q_heads, batch, max_len) -> int:
    return lib().forge_attn_paged_workspace_bytes(C.byref(cache), q_heads, batch, max_len)


def forge_attn_paged(cache: PagedCache, q, out, lengths, table, max_len, scale=None, workspace=None, layer=0):
    """q [B,Hq,dh] view; out [B,Hq*dh]; request b attends to its first lengths[b] rows (none: zeros), in the pages table[b] names."""
    B, H, dh = q.shape
    if dh != cache.head_dim or out.shape != (B, H * dh) or lengths is None or table.dim() != 2 or table.shape[0] != B:
        raise ValueError("q must be [B, Hq, %d], out [B, Hq * %d], table [B, cols]" % (cache.head_dim, cache.head_dim))
    _cache_dt(cache, q, out)
    (sb, sh, sd), d = q.stride(), _device()
    _here(cache, d)
    if q.get_device() != d or (sd != 1 and dh != 1):
        _refuse(q.get_device(), d, "forge needs [request, head, head_dim] GPU tensors with a dense last axis")
    view = Heads(q.data_ptr(), sb, 0, sh)
    wp, wb = _ws_at(workspace, d)
    _check(lib().forge_attn_paged(C.byref(cache), layer, C.byref(view), _at(out, d), _vector(lengths, B, "lengths", d),
                                  _vector(table, B * table.shape[1], "table", d), table.shape[1], H, B, max_len,
                                  dh ** -0.5 if scale is None else scale, wp, wb, _stream(d)), "forge_attn_paged")
    return out


def make_adapters(a, b, scale=None, part_end=None) -> Adapters:
    """a [n, parts * rank, K], b [n, N, rank], scale fp32 [n] or None; part_end: the columns at which the parts of N end (None: one).
    The struct keeps them alive."""
    n, N, rank = b.shape
    ends = [N] if part_end is None else [int(e) for e in part_end]
    if not 1 <= len(ends) <= 4 or a.shape[0] != n or a.shape[1] != len(ends) * rank or a.dtype != b.dtype:
        raise ValueError("a must be [n, parts * rank, K] and b [n, N, rank], 1 to 4 parts")
    if scale is not None and (scale.dtype != torch.float32 or scale.shape != (n,)):
        raise ValueError("scale must be fp32 of shape (%d,)" % n)
    return _keeping(Adapters(_dt(a), n, rank, a.shape[2], N, len(ends), (C.c_int * 4)(*ends), _p(a), _p(b), _p(scale)), (a, b, scale))


def forge_adapters_workspace_bytes(adapters: Adapters, M) -> int:
    return lib().forge_adapters_workspace_bytes(C.byref(adapters), M)


def forge_adapters_add(adapters: Adapters, x, base, y, ids, workspace=None):
    """y[m, :N] = base[m, :N] + the adapter ids[m] of x[m] (none where it is outside the range); y may be base, and both wider than N."""
    (M, K), d = x.shape, _device()
    _here(adapters, d)
    if K != adapters.K or base.shape != y.shape or y.shape[0] != M or ids is None:
        raise ValueError("x must be [M, %d], base and y [M, at least %d]" % (adapters.K, adapters.N))
    if not x.dtype == base.dtype == y.dtype or _dt(x) != adapters.dt:
        raise ValueError("x, base, y and the adapters must agree in dtype")
    wp, wb = _ws_at(workspace, d)
    _check(lib().forge_adapters_add(C.byref(adapters), _at(x, d), _at(base, d), _at(y, d), _vector(ids, M, "ids", d), M, y.shape[1], wp, wb,
                                    _stream(d)), "forge_adapters_add")
    return y


# ---------------------------------------------------------------------------------------------
# Static buffer plan (host arrays in, host arrays out) and the compiled executor.


def _ints(values):
    return (C.c_int * max(1, len(values)))(*values)


def forge_plan_liveness(out_reg: Sequence[int], in_lists: Sequence[Sequence[int]], n_regs: int):
    """Program = per instruction an output register (-1: none) and the registers it reads.
    Returns (start, end) lists, -1 for registers never mentioned."""
    n = len(out_reg)
    begin, flat = [0], []
    for ins in in_lists:
        flat.extend(ins)
        begin.append(len(flat))
    start, end = _ints([0] * n_regs), _ints([0] * n_regs)
    _check(lib().forge_plan_liveness(n, _ints(out_reg), _ints(begin), _ints(flat), n_regs, start, end),
           "forge_plan_liveness")
    return list(start)[:n_regs], list(end)[:n_regs]


def forge_plan_dead_after(end: Sequence[int], n_instr: int) -> Dict[int, list]:
    live = sum(1 for e in end if e >= 0)
    begin, regs = _ints([0] * (n_instr + 1)), _ints([0] * live)
    _check(lib().forge_plan_dead_after(len(end), _ints(end), n_instr, begin, regs), "forge_plan_dead_after")
    return {j: list(regs[begin[j]:begin[j + 1]]) for j in range(n_instr) if begin[j + 1] > begin[j]}


def forge_plan_linear_scan(start: Sequence[int], end: Sequence[int]):
    n = len(start)
    buf, m = _ints([0] * n), C.c_int(0)
    _check(lib().forge_plan_linear_scan(n, _ints(start), _ints(end), buf, C.byref(m)), "forge_plan_linear_scan")
    return list(buf)[:n], m.value


def forge_plan_workspace(start: Sequence[int], end: Sequence[int], nbytes: Sequence[int]):
    """Returns (offset per register, total bytes, number of buffers); offset -1 where start < 0."""
    n = len(start)
    sizes = (C.c_size_t * max(1, n))(*nbytes)
    off = (C.c_size_t * max(1, n))()
    total, m = C.c_size_t(0), C.c_int(0)
    _check(lib().forge_plan_workspace(n, _ints(start), _ints(end), sizes, off, C.byref(total), C.byref(m)),
           "forge_plan_workspace")
    none = C.c_size_t(-1).value
    return [-1 if o == none else o for o in list(off)[:n]], total.value, m.value


class CompiledModel:
    """Handle of forge_compile_model for one fixed (batch, q_len, pos0, kv_cap).  `bind` records
    the HIP graph on a non-default stream, `run` replays it.  Keeps the descriptor (and through
    it nothing else) alive: the caller keeps the weight tensors alive."""

    def __init__(self, model: ModelDesc, batch: int, q_len: int, pos0: int, kv_cap: int):
        self._h = C.c_void_p(None)
        self._model = model
        _check(lib().forge_compile_model(C.byref(model), batch, q_len, pos0, kv_cap, C.byref(self._h)),
               "forge_compile_model")
        self._bound = None

    def close(self):
        if self._h:
            lib().forge_compiled_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self) -> int:
        return lib().forge_compiled_workspace_bytes(self._h)

    def counts(self):
        """(instructions, registers, register reads, buffers)"""
        a, b, c, d = C.c_int(0), C.c_int(0), C.c_int(0), C.c_int(0)
        _check(lib().forge_compiled_counts(self._h, C.byref(a), C.byref(b), C.byref(c), C.byref(d)),
               "forge_compiled_counts")
        return a.value, b.value, c.value, d.value

    def program(self):
        """(ops, out_reg, in_lists, reg_bytes, reg_offset)"""
        ni, nr, nreads, _ = self.counts()
        op, out, begin, regs = _ints([0] * ni), _ints([0] * ni), _ints([0] * (ni + 1)), _ints([0] * nreads)
        nb, off = (C.c_size_t * max(1, nr))(), (C.c_size_t * max(1, nr))()
        _check(lib().forge_compiled_program(self._h, op, out, begin, regs, nb, off), "forge_compiled_program")
        ins = [list(regs[begin[j]:begin[j + 1]]) for j in range(ni)]
        return list(op)[:ni], list(out)[:ni], ins, list(nb)[:nr], list(off)[:nr]

    def bind(self, inp, out, k_cache, v_cache, workspace, stream: "torch.cuda.Stream"):
        wp, wb = _ws(workspace)
        _check(lib().forge_compiled_bind(self._h, _p(inp), _p(out), _p(k_cache), _p(v_cache), wp, wb,
                                         C.c_void_p(stream.cuda_stream)), "forge_compiled_bind")
        self._bound = (inp, out, k_cache, v_cache, workspace)     # keep the tensors alive
        return self

    def bind_decode(self, inp, out, k_cache, v_cache, seq_pos, workspace, stream: "torch.cuda.Stream"):
        wp, wb = _ws(workspace)
        _check(lib().forge_compiled_bind_decode(self._h, _p(inp), _p(out), _p(k_cache), _p(v_cache), _p(seq_pos),
                                                wp, wb, C.c_void_p(stream.cuda_stream)), "forge_compiled_bind_decode")
        self._bound = (inp, out, k_cache, v_cache, seq_pos, workspace)
        return self

    def run(self, stream: "torch.cuda.Stream"):
        _check(lib().forge_compiled_run(self._h, C.c_void_p(stream.cuda_stream)), "forge_compiled_run")
