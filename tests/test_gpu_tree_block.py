"""A decoder layer over drafted trees: against the oracle's layer fed branch by branch, against its own operators called one by one,
and a generation loop against one-by-one decoding."""
import numpy as np
import pytest
import torch

from oracle import forge_oracle as O
from paper_2604_16498_amd import binding as F
from paper_2604_16498_amd import inputs as I
from paper_2604_16498_amd import tree_decode as T
from tree_inputs import ancestor_bits, cache_arrays, depths, gpu, parents, signed
from util import check, dev, dev_dict, host

pytestmark = pytest.mark.gpu

LLAMA = I.BlockShape(512, 8, 2, 64, 704, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=500000.0, has_bias=False)
WIDE = I.BlockShape(512, 8, 2, 128, 1024, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=10000.0, has_bias=False)
GPT = I.BlockShape(384, 6, 6, 64, 1536, has_bias=True)


def ints(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def rope_of(sh):
    if not sh.use_rope:
        return None
    inc, factor = F.forge_rope_increments(sh.rope_base, sh.head_dim)
    return F.make_rope_desc(inc.cuda(), "half", factor)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("name,n,pos", [("llama", 1, [5, 0, 40]), ("llama", 13, [70, 3]), ("wide", 24, [33]), ("gpt", 9, [12, 100])])
def test_layer_follows_every_branch(name, n, pos, bf16):
    sh = {"llama": LLAMA, "wide": WIDE, "gpt": GPT}[name]
    rng = np.random.default_rng(n)
    B, cap = len(pos), max(pos) + n + 5
    w = I.block_weights(sh, 99, n, bf16=bf16, random_affine=True)
    x = I.normal(99, n, "x", (B, n, sh.d_model), 1.0, bf16=bf16)
    (k, v, _, _), (rk, rv) = cache_arrays(rng, "bf16" if bf16 else "fp32", (1, B, sh.kv_heads, cap, sh.head_dim))
    tw = dev_dict(w, bf16)
    desc = F.make_block_desc(sh, tw)
    trees = [parents(rng, n) for _ in range(B)]
    cache = F.make_kv_cache(k, v)
    ws = F.workspace(F.forge_decoder_block_tree_workspace_bytes(desc, cache, n, max(pos)))
    out = torch.empty(B, n, sh.d_model, dtype=k.dtype, device="cuda")
    where = ints(pos)[:, None] + ints([depths(t) for t in trees])
    F.forge_decoder_block_tree(desc, cache, dev(x, bf16), out, ints(pos), max(pos), ws, rope=rope_of(sh), positions=where,
                               visible=ints(signed([ancestor_bits(t) for t in trees]), torch.int64))
    got, ref = [], []
    for b in range(B):
        leaves = set(range(n)) - set(trees[b])
        for leaf in leaves:
            branch, at = [], leaf
            while at >= 0:
                branch.insert(0, at)
                at = trees[b][at]
            room = np.zeros((1, sh.kv_heads, pos[b] + len(branch), sh.head_dim))
            kc, vc = room.copy(), room.copy()
            kc[0, :, :pos[b]], vc[0, :, :pos[b]] = rk[0, b, :, :pos[b]], rv[0, b, :, :pos[b]]
            ref.append(O.decoder_block(sh, w, x[b:b + 1, branch], kc, vc, pos0=pos[b])[0])
            got.append(out[b, branch])
    check(torch.cat(got), np.concatenate(ref), bf16, "tree layer %s n=%d" % (name, n), chain=True)


@pytest.mark.parametrize("w8", [False, True])
@pytest.mark.parametrize("store", ["int8", "fp8", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 40])
def test_layer_is_its_operators(n, store, w8):
    """The launch list gives what the public operators give one by one; x_out may be x_in."""
    sh = I.BlockShape(512, 8, 2, 64, 768, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=10000.0, has_bias=False)
    rng = np.random.default_rng(n)
    B, pos, cap = 3, [600, 17, 0], 700
    w = dev_dict(I.block_weights(sh, 98, n, bf16=True, random_affine=True), True)
    if w8:
        for name in ("qkv", "o", "up", "down"):
            w["w_" + name], w["s_" + name] = F.forge_quantize_int8(w["w_" + name])
    desc = F.make_block_desc(sh, w)
    x = dev(I.normal(98, n, "x", (B, n, sh.d_model), 1.0, bf16=True), True)
    arrays, _ = cache_arrays(rng, store, (2, B, sh.kv_heads, cap, sh.head_dim))
    twin = [None if a is None else a.clone() for a in arrays]
    one, two = F.make_kv_cache(*arrays), F.make_kv_cache(*twin)
    vis = ints(signed([ancestor_bits(parents(rng, n)) for _ in range(B)]), torch.int64)
    seq = ints(pos)
    ws = F.workspace(F.forge_decoder_block_tree_workspace_bytes(desc, one, n, 600))
    y = x.clone()
    F.forge_decoder_block_tree(desc, one, y, y, seq, 600, ws, rope=rope_of(sh), visible=vis, layer=1)

    rows, d, heads = B * n, sh.d_model, sh.q_heads + 2 * sh.kv_heads

    def linear(a, name, act="none", residual=None, cols=None):
        o = torch.empty(rows, cols or d, dtype=torch.bfloat16, device="cuda")
        k_dim = a.shape[1]
        if w8:
            space = F.workspace(F.forge_gemm_w8_workspace_bytes(rows, o.shape[1], k_dim, act))
            return F.forge_gemm_w8(a, w["w_" + name], w["s_" + name], None, residual, o, act=act, workspace=space)
        space = F.workspace(F.forge_gemm_workspace_bytes(rows, o.shape[1], k_dim, act, torch.bfloat16))
        return F.forge_gemm_bias_gelu(a, w["w_" + name], None, residual, o, act=act, workspace=space)

    def norm(a, g):
        o = torch.empty_like(a)
        F.forge_residual_norm(a, None, w[g], None, None, o, eps=sh.eps, kind="rmsnorm")
        return o
    flat = x.view(rows, d)
    qkv = linear(norm(flat, "norm1_g"), "qkv", cols=heads * sh.head_dim).view(B, n, heads, sh.head_dim)
    q, kk, vv = qkv[:, :, :sh.q_heads], qkv[:, :, sh.q_heads:sh.q_heads + sh.kv_heads], qkv[:, :, sh.q_heads + sh.kv_heads:]
    F.forge_kv_append(two, kk, vv, seq, 600, rope=rope_of(sh), q=q, q_out=q, layer=1)
    o = torch.empty(B, n, sh.q_heads * sh.head_dim, dtype=torch.bfloat16, device="cuda")
    F.forge_attn_tree(two, q, o, seq, 600, visible=vis, workspace=F.workspace(F.forge_attn_tree_workspace_bytes(two, sh.q_heads, n, 600)), layer=1)
    for a, b in zip(arrays, twin):
        assert a is None or torch.equal(a.view(torch.uint8) if a.element_size() == 1 else a, b.view(torch.uint8) if b.element_size() == 1 else b)
    h = linear(o.view(rows, -1), "o", residual=flat)
    u = linear(norm(h, "norm2_g"), "up", act="swiglu", cols=sh.d_ff)
    want = linear(u, "down", residual=h)
    # (a decode-sized layer normalises the fp32 sum before it is rounded: an ulp of bf16 here and there)
    check(y, host(want).reshape(y.shape), True, "layer by operators n=%d" % n, chain=True)


def test_a_branch_is_what_its_tokens_give_one_by_one():
    """After a commit the cache holds what feeding the accepted tokens singly leaves in it, and attention over it agrees."""
    sh = LLAMA
    rng = np.random.default_rng(3)
    n, pos, cap = 8, 50, 80
    w = dev_dict(I.block_weights(sh, 97, 0, bf16=True, random_affine=True), True)
    desc = F.make_block_desc(sh, w)
    x = dev(I.normal(97, 0, "x", (1, n, sh.d_model), 1.0, bf16=True), True)
    arrays, _ = cache_arrays(rng, "int8", (1, 1, sh.kv_heads, cap, sh.head_dim))
    twin = [a.clone() for a in arrays]
    one, two = F.make_kv_cache(*arrays), F.make_kv_cache(*twin)
    tree = [-1, 0, 0, 2, 1, 3, 3, 5]
    branch = [0, 2, 3, 5, 7]
    ws = F.workspace(max(F.forge_decoder_block_tree_workspace_bytes(desc, one, m, cap - m) for m in (1, n)))
    out = torch.empty_like(x)
    F.forge_decoder_block_tree(desc, one, x, out, ints([pos]), pos, ws, rope=rope_of(sh), positions=ints([[pos + d for d in depths(tree)]]),
                               visible=ints(signed([ancestor_bits(tree)]), torch.int64))
    F.forge_kv_commit(one, ints([branch + [0] * (n - len(branch))]), ints([len(branch)]), ints([pos]), pos)
    single = torch.empty_like(x)
    for i, t in enumerate(branch):
        F.forge_decoder_block_tree(desc, two, x[:, t:t + 1].contiguous(), single[:, t:t + 1], ints([pos + i]), pos + i, ws, rope=rope_of(sh))
    check(out[:, branch], host(single[:, branch]), True, "branch against single tokens", chain=True)
    k, v = (torch.empty(2, 1, sh.kv_heads, len(branch), sh.head_dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for i, c in enumerate((one, two)):
        F.forge_kv_read(c, k[i], v[i], max_pos=pos)
    # both sides project the same rows, by kernels for one row and for eight: a bf16 rounding apart, and a step of the codes (1/127 of the
    # row's largest) where that crosses a boundary
    for a in (k, v):
        a = host(a)
        assert (np.abs(a[0] - a[1]) <= 1.1 / 127 * np.abs(a).max(-1, keepdims=True)[0] + 2.0 ** -8 * np.abs(a[1])).all()


@pytest.mark.parametrize("store", ["int8", "same"])
def test_generation_with_trees_gives_the_greedy_tokens(store):
    sh = I.BlockShape(256, 4, 2, 64, 512, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=10000.0, has_bias=False)
    weights, top = T.random_model(sh, 2, 211, seed=5)
    ids = torch.randint(0, 211, (3, 90), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    lengths = [90, 40, 1]
    make = lambda: T.TreeDecoder(sh, weights, top, 3, 256, store=store, scaling="linear", by=2.0)
    model = make()
    plain = T.generate(model, model.prompt(ids, lengths), 24, lambda tokens: ([], []))
    assert all(len(p) == 25 for p in plain)
    model = make()
    first = model.prompt(ids, lengths)
    assert first.tolist() == [p[0] for p in plain]

    def draft(tokens):
        here = [p for p in plain if p[:len(tokens)] == tokens]
        right = here[0][len(tokens):len(tokens) + 3] if here else []
        wrong = [(t + 7) % 211 for t in right]
        # wrong first, so that the accepted rows have to move; the right branch with a wrong leaf in between
        ids_, par = list(wrong), [0] + list(range(1, len(wrong))) if wrong else []
        at = 0
        for t in right:
            ids_ += [(t + 1) % 211, t]
            par += [at, at]
            at = len(ids_)
        return ids_, par
    trees = T.generate(model, first, 6, draft)
    for a, b in zip(plain, trees):
        m = min(len(a), len(b))
        assert a[:m] == b[:m] and len(b) == 25          # three drafts and one choice a pass
    assert model.seq_pos.tolist() == [l + 24 for l in lengths]


def test_decoder_refuses_what_does_not_fit():
    sh = I.BlockShape(256, 4, 2, 64, 512, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=10000.0, has_bias=False)
    weights, top = T.random_model(sh, 1, 50)
    model = T.TreeDecoder(sh, weights, top, 1, 12, drafts=4)
    ids = torch.zeros(1, 10, dtype=torch.int32, device="cuda")
    for bad in ([11], [0], [5, 5]):
        with pytest.raises(ValueError):
            model.prompt(ids, bad)
    model.prompt(ids, [10])
    with pytest.raises(ValueError):
        model.prompt(ids, [10])
    for tree in ([-1, 0, 1, 2, 3], [-1, 0, 2, 1], [0, 0], [-1, -1], [-1, 0, 0]):      # too many, parents last, no root, two, no room
        with pytest.raises(ValueError):
            model.verify(ids[:, :len(tree)], [tree])
    model.verify(ids[:, :2], [[-1, 0]])


def test_layer_refusals():
    sh = LLAMA
    w = dev_dict(I.block_weights(sh, 96, 0, bf16=True), True)
    desc = F.make_block_desc(sh, w)
    arrays, _ = cache_arrays(np.random.default_rng(0), "int8", (1, 2, sh.kv_heads, 64, sh.head_dim))
    cache = F.make_kv_cache(*arrays)
    ws = F.workspace(F.forge_decoder_block_tree_workspace_bytes(desc, cache, 4, 30))
    x = torch.zeros(2, 4, sh.d_model, dtype=torch.bfloat16, device="cuda")
    call = lambda **kw: F.forge_decoder_block_tree(desc, kw.get("cache", cache), x, x, ints([3, 4]), kw.get("mp", 30), kw.get("ws", ws), rope=kw.get("rope", rope_of(sh)))
    call()
    other, _ = cache_arrays(np.random.default_rng(0), "int8", (1, 2, sh.kv_heads, 64, 128))
    for kw, status in ((dict(rope=None), 1), (dict(mp=61), 1), (dict(ws=None), 1), (dict(ws=ws[:256]), 3), (dict(cache=F.make_kv_cache(*other)), 1)):
        with pytest.raises(F.ForgeError) as e:
            call(**kw)
        assert e.value.status == status, kw
    with pytest.raises(ValueError):
        F.forge_decoder_block_tree(desc, cache, x.float(), x.float(), ints([3, 4]), 30, ws, rope=rope_of(sh))
