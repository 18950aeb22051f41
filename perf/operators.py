"""The operators of serving drafted tokens over a quantised cache, whose speed is measured beside their plain forms.

A case is a dict of plain values; `listed` gives the fixed ones and `draw` more of the same ranges.  Operators:
  rope       rotary positions of the new rows: both pairings, the whole head or its first part, scaled for long contexts
  append     the new rows of a step or a prompt: q and k rotated, k and v quantised into the cache; the rows just written
             are read back
  read       a history read back from the quantised cache, as a prompt's attention takes it
  attention  a tree of drafted tokens (or one token) per sequence over a ragged cache
  commit     the accepted branch's rows moved together in the caches of all layers
Where `own` is false they are computed in elementary torch operations, in 32 bits and rounded once at the end; where it is true
by the calls of paper_2604_16498_amd.binding.
"""
import math
import random

import torch

own = False

# query heads, key / value heads, head size, rotary base, layers of the shapes that this repository serves
SHAPES = {
    "gpt2s": (12, 12, 64, 10000.0, 12),
    "1p3b": (16, 16, 128, 10000.0, 24),
    "8b": (32, 8, 128, 500000.0, 32),
}
SCALINGS = ("none", "linear", "base", "bands", "ramp")
SCALE_BY, CONTEXT = 8.0, 8192          # contexts eight times as long as the 8192 positions trained on
TOP = {"int8": 127.0, "fp8": 448.0}    # the largest code of a quantised row
MOST_PAIRS = 16 * 64 * 8255            # sequences x drafted tokens x rows of the largest attention


def rope(name, shape, batch, seq, pos=0, dtype="bf16", style="half", part=1, scaling="none"):
    """pos: largest position that the new rows follow.  part: the first 1 / part of each head turns."""
    c = {"kind": "rope", "shape": shape, "batch": batch, "seq": seq, "pos": pos, "dtype": dtype, "style": style, "part": part,
         "scaling": scaling}
    return dict(c, name=name) if name else c


def append(name, shape, batch, seq, pos, store, tree=False, style="half", part=1, scaling="none"):
    """store: "int8", "fp8" or "same" (bf16).  tree: the new rows are a tree of drafts, their positions its depths."""
    c = {"kind": "append", "shape": shape, "batch": batch, "seq": seq, "pos": pos, "store": store, "tree": tree, "style": style,
         "part": part, "scaling": scaling}
    return dict(c, name=name) if name else c


def read(name, shape, batch, rows, store):
    c = {"kind": "read", "shape": shape, "batch": batch, "rows": rows, "store": store}
    return dict(c, name=name) if name else c


def attention(name, shape, batch, seq, pos, store):
    """seq: drafted tokens of each sequence.  store: "int8", "fp8", "same" (bf16) or "fp32"."""
    c = {"kind": "attention", "shape": shape, "batch": batch, "seq": seq, "pos": pos, "store": store}
    return dict(c, name=name) if name else c


def commit(name, shape, layers, batch, seq, pos, store):
    c = {"kind": "commit", "shape": shape, "layers": layers, "batch": batch, "seq": seq, "pos": pos, "store": store}
    return dict(c, name=name) if name else c


def listed():
    return [
        # a decode step of the small model in full precision, a quarter of each head turned pairwise: latency
        rope("rope_gpt2s_fp32_b3_s1", "gpt2s", 3, 1, pos=640, dtype="fp32", style="interleaved", part=4, scaling="linear"),
        # a long prompt of the large model far into a context stretched by bands: bandwidth
        rope("rope_8b_b1_s4096_bands", "8b", 1, 4096, pos=30011, scaling="bands"),
        # a drafting step of a serving batch: 13 drafts for each of 24 sequences of different lengths
        append("append_8b_int8_b24_tree13", "8b", 24, 13, 1500, "int8", tree=True, scaling="bands"),
        # a prompt of the middle model written into an fp8 cache
        append("append_1p3b_fp8_b4_s2048", "1p3b", 4, 2048, 0, "fp8", style="interleaved"),
        # the short history of three chats with the small model
        read("read_gpt2s_fp8_b3_r77", "gpt2s", 3, 77, "fp8"),
        # the next turn of a conversation over a long document: its whole history
        read("read_8b_int8_b4_r8191", "8b", 4, 8191, "int8"),
        # one token of one sequence of the small model: latency
        attention("attention_gpt2s_b1_n1", "gpt2s", 1, 1, 333, "same"),
        # throughput serving: one token for each of 64 sequences of different lengths
        attention("attention_8b_int8_b64_n1", "8b", 64, 1, 2048, "int8"),
        # few users with long documents, trees of 26 drafts
        attention("attention_8b_fp8_b5_tree26", "8b", 5, 26, 8191, "fp8"),
        # throughput serving with the widest trees, 16 bits: as much matrix work as reading
        attention("attention_8b_b16_tree64", "8b", 16, 64, 8191, "same"),
        # one chat of the small model, after each verification
        commit("commit_gpt2s_b1_tree5", "gpt2s", 12, 1, 5, 333, "same"),
        # a serving batch of the large model, the caches of a stage of 8 layers
        commit("commit_8b_int8_b24_tree26", "8b", 8, 24, 26, 1023, "int8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "read", "attention", "attention", "attention", "commit"])
    shape = rng.choice(list(SHAPES))
    style, part, scaling = rng.choice(["half", "interleaved"]), rng.choice([1, 1, 2, 4]), rng.choice(SCALINGS)
    if kind == "rope":
        batch = _log_int(rng, 1, 64)
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        most = (4096 if shape == "8b" else 8192) // (2 if dtype == "fp32" else 1)
        return rope("", shape, batch, _log_int(rng, 1, most // batch), _log_int(rng, 1, 100000), dtype, style, part, scaling)
    store = rng.choice(["int8", "fp8", "same"])
    if kind == "append":
        batch = _log_int(rng, 1, 64)
        tree = rng.random() < 0.6
        seq = _log_int(rng, 1, 64) if tree else _log_int(rng, 1, 8192 // batch)
        return append("", shape, batch, seq, _log_int(rng, 1, 64 * 2048 // batch if batch > 15 else 8191), store, tree, style, part, scaling)
    if kind == "read":
        batch = _log_int(rng, 1, 64)
        top = 4 * 8191 if shape == "8b" else 4 * 4095        # the 8b shape has half the key / value heads of the 1p3b one
        return read("", shape, batch, _log_int(rng, 1, min(8191, top // batch)), rng.choice(["int8", "fp8"]))
    if kind == "commit":
        layers, batch = rng.randint(1, 8), _log_int(rng, 1, 24)
        return commit("", shape, layers, batch, rng.randint(2, 64), _log_int(rng, 16, 1000), store)
    store = rng.choice(["int8", "int8", "fp8", "fp8", "same", "fp32"])
    batch = _log_int(rng, 1, 64)
    pos = _log_int(rng, 16, min(8191, 64 * (1024 if shape == "1p3b" else 2048) // batch))     # key / value heads: 16, 8
    seq = 1 if rng.random() < 0.3 else _log_int(rng, 2, 64)
    if store == "fp32":          # full precision: the small model, short contexts
        return attention("", "gpt2s", min(batch, 8), min(seq, 32), min(pos, 1000), store)
    return attention("", shape, batch, max(1, min(seq, MOST_PAIRS // (batch * (pos + 64)))), pos, store)


# ---------------------------------------------------------------------------------------------
# inputs


def _lengths(case):
    """Cached rows of every sequence: between a quarter of the longest and all of it."""
    b, top = case["batch"], case["pos"]
    return [top - (3 * top * (b - 1 - i)) // (4 * max(1, b - 1)) for i in range(b)]


def _trees(case, seed):
    """Per sequence the parent of every drafted token (-1: it follows the cached rows): a main chain with branches."""
    r, got = random.Random(seed), []
    for _ in range(case["batch"]):
        got.append([t - 1 if r.random() < 0.5 else r.randint(max(-1, t - 5), t - 1) for t in range(case["seq"])])
    return got


def _ancestors(parents):
    """(bits of the drafts that each one sees, itself among them, as signed 64-bit numbers; depths)."""
    bits, depth = [], []
    for t, p in enumerate(parents):
        bits.append((bits[p] if p >= 0 else 0) | 1 << t)
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return [b - (1 << 64) if b >> 63 else b for b in bits], depth


def _frequencies(case, np_pi=math.pi):
    """Radians a position of every pair, and what cos and sin are multiplied by: the definition."""
    _, _, dh, base, _ = SHAPES[case["shape"]]
    r, s, kind = dh // case["part"], SCALE_BY, case["scaling"]
    if kind == "base":
        base *= s ** (r / (r - 2))
    theta = [base ** (-2.0 * i / r) for i in range(r // 2)]
    if kind == "linear":
        theta = [t / s for t in theta]
    if kind == "bands":          # kept over 4 turns in the trained context, divided below 1, blended between
        for i, t in enumerate(theta):
            g = min(1.0, max(0.0, (CONTEXT * t / (2 * np_pi) - 1.0) / 3.0))
            theta[i] = t * (g + (1 - g) / s)
    if kind == "ramp":           # the same, but a line over the pairs between 32 turns and 1
        pair = lambda turns: r * math.log(CONTEXT / (turns * 2 * np_pi)) / (2 * math.log(base))
        lo, hi = max(0, math.floor(pair(32.0))), min(r - 1, math.ceil(pair(1.0)))
        for i, t in enumerate(theta):
            g = 1.0 - min(1.0, max(0.0, (i - lo) / max(0.001, hi - lo)))
            theta[i] = t * (g + (1 - g) / s)
        return theta, 0.1 * math.log(s) + 1.0
    return theta, 1.0


def _quantised(x, store):
    """Rows of x as (codes, scales): what an earlier step of the program left in the cache."""
    top = x.float().abs().amax(-1)
    scale = torch.where(top / TOP[store] < 2.0 ** -126, 1.0, top / TOP[store])
    y = x.float() / scale[..., None]
    return (torch.round(y).to(torch.int8) if store == "int8" else y.to(torch.float8_e4m3fn)), scale


def _caches(shape, store, normal):
    """k and v of the given shape with their scales (None where rows are held as they are)."""
    st = {}
    for name in ("k", "v"):
        x = normal(shape, torch.float32 if store == "fp32" else torch.bfloat16)
        st[name + "_cache"], st[name + "_scale"] = _quantised(x, store) if store in TOP else (x, None)
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    hq, hkv, dh, _, _ = SHAPES[case["shape"]]
    B, kind = case["batch"], case["kind"]

    def normal(shape, dt=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def ints(v, dt=torch.int32):
        return torch.tensor(v, dtype=dt, device="cuda")

    st = {"case": case}
    if kind in ("rope", "append"):
        theta, st["factor"] = _frequencies(case)
        # the plan that a program keeps: each pair's turn a position, in units of 2^-64 of a full turn
        st["increments"] = ints([round(t / (2 * math.pi) * 2.0 ** 64) for t in theta], torch.int64)
    if kind == "read":
        cap = (case["rows"] + 63) // 64 * 64
        st.update(_caches((B, hkv, cap, dh), case["store"], normal))
        st["k_out"], st["v_out"] = (torch.empty(B, hkv, case["rows"], dh, device="cuda", dtype=torch.bfloat16) for _ in range(2))
        return st
    n, pos = case["seq"], case["pos"]
    lengths = _lengths(case)
    random.Random(seed).shuffle(lengths)
    st["seq_pos"] = ints(lengths)
    trees = _trees(case, seed) if kind in ("attention", "commit") or case.get("tree") else None
    if kind in ("rope", "append"):
        steps = [_ancestors(t)[1] for t in trees] if trees else [list(range(n))] * B
        st["positions"] = st["seq_pos"][:, None] + ints(steps)
        # q, k and v as the projection leaves them: one row a token, all heads side by side
        dt = torch.float32 if case.get("dtype") == "fp32" else torch.bfloat16
        rows = normal((B, n, hq + 2 * hkv, dh), dt)
        if kind == "rope":
            st["x"] = rows[:, :, :hq + hkv]
            st["y"] = torch.empty(B, n, hq + hkv, dh, device="cuda", dtype=dt)
            return st
        st["q"], st["k"], st["v"] = rows[:, :, :hq], rows[:, :, hq:hq + hkv], rows[:, :, hq + hkv:]
    cap = (pos + n + 63) // 64 * 64
    layers = (case["layers"],) if kind == "commit" else ()
    st.update(_caches(layers + (B, hkv, cap, dh), case["store"], normal))
    if kind == "append":
        st["q_out"] = torch.empty(B, n, hq, dh, device="cuda", dtype=torch.bfloat16)
        st["k_out"], st["v_out"] = (torch.empty(B, hkv, n, dh, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    if kind == "attention":
        dt = st["k_cache"].dtype if case["store"] == "fp32" else torch.bfloat16
        st["q"] = normal((B, n, hq, dh), dt)
        st["visible"] = ints([_ancestors(t)[0] for t in trees], torch.int64)
        st["out"] = torch.empty(B, n, hq * dh, device="cuda", dtype=dt)
    if kind == "commit":
        path, taken = [], []
        for i, t in enumerate(trees):      # from a drafted token back to the root: the branch that was accepted
            at, branch = random.Random(seed + i).randrange(-1, n), []
            while at >= 0:
                branch.insert(0, at)
                at = t[at]
            taken.append(len(branch))
            path.append(branch + [0] * (n - len(branch)))
        st["path"], st["taken"] = ints(path), ints(taken)
    return st


# ---------------------------------------------------------------------------------------------
# the plain forms


def _turn(x, st):
    """x [B, n, heads, dh] in 32 bits, rotated."""
    case = st["case"]
    # positions times increments wrap at whole turns; the rest counts from the nearest quarter
    phase = st["positions"].long()[:, :, None] * st["increments"]
    quarter = ((phase >> 61) + 1) >> 1
    angle = (phase - (quarter << 62)).float() * (2 * math.pi / 2.0 ** 64)
    c, s = torch.cos(angle), torch.sin(angle)
    odd = (quarter & 1).bool()
    c, s = torch.where(odd, -s, c), torch.where(odd, c, s)
    sign = torch.where((quarter & 2).bool(), -st["factor"], st["factor"])
    c, s = (c * sign)[:, :, None], (s * sign)[:, :, None]
    r = x.shape[-1] // case["part"]
    if case["style"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., r:]], -1)


def _plain_append(st):
    case = st["case"]
    B, n = case["batch"], case["seq"]
    rows = (st["seq_pos"].long()[:, None] + torch.arange(n, device="cuda"))[:, None].expand(B, st["k"].shape[2], n)
    for name, x in (("k", _turn(st["k"].float(), st)), ("v", st["v"].float())):
        x = x.transpose(1, 2)
        cache, scale, out = st[name + "_cache"], st[name + "_scale"], st[name + "_out"]
        wide = rows[..., None].expand(x.shape)
        if scale is None:
            cache.scatter_(2, wide, x.to(cache.dtype))
            out.copy_(cache.gather(2, wide))
            continue
        codes, s = _quantised(x, case["store"])
        cache.view(torch.int8).scatter_(2, wide, codes.view(torch.int8))
        scale.scatter_(2, rows, s)
        back = cache.view(torch.int8).gather(2, wide).view(cache.dtype)
        out.copy_(back.float() * scale.gather(2, rows)[..., None])
    st["q_out"].copy_(_turn(st["q"].float(), st))


def _seen(st, rows):
    """[B, n, rows]: which cache rows each drafted token attends to."""
    at = torch.arange(rows, device="cuda") - st["seq_pos"].long()[:, None]
    drafted = (at >= 0) & (at < st["case"]["seq"])
    bit = st["visible"][:, :, None] >> at.clamp(0, 63)[:, None] & 1
    return (at < 0)[:, None] | drafted[:, None] & bit.bool()


def _plain_attention(st):
    case = st["case"]
    B, n, hq, dh = st["q"].shape
    hkv, rows = st["k_cache"].shape[1], case["pos"] + n
    k, v = (st[x + "_cache"][:, :, :rows].float() for x in ("k", "v"))
    if st["k_scale"] is not None:
        k, v = k * st["k_scale"][:, :, :rows, None], v * st["v_scale"][:, :, :rows, None]
    q = st["q"].float().view(B, n, hkv, hq // hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, hkv, -1, dh)
    s = torch.matmul(q, k.transpose(2, 3)) * dh ** -0.5
    s = s.view(B, hkv, hq // hkv, n, rows).masked_fill(~_seen(st, rows)[:, None, None], -torch.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True))
    o = torch.matmul(p.view(B, hkv, -1, rows), v).view(B, hkv, hq // hkv, n, dh) / p.sum(-1, keepdim=True)
    st["out"].copy_(o.permute(0, 3, 1, 2, 4).reshape(B, n, hq * dh))


def _moves(st):
    """(from, to): cache rows, [B, n]; entries past the accepted ones move a row onto itself."""
    step = torch.arange(st["case"]["seq"], device="cuda")
    to = st["seq_pos"].long()[:, None] + step
    return torch.where(step < st["taken"][:, None], st["seq_pos"].long()[:, None] + st["path"], to), to


def _plain_commit(st):
    src, dst = _moves(st)
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        x = st[name]
        if x is None:
            continue
        x = (x.view(torch.int8) if x.element_size() == 1 else x)
        x = x if x.dim() == 5 else x[..., None]
        shape = x.shape[:3] + (src.shape[1], x.shape[4])
        wide = lambda i: i[None, :, None, :, None].expand(shape)
        x.scatter_(3, wide(dst), x.gather(3, wide(src)))


def _outputs(st):
    kind = st["case"]["kind"]
    if kind == "rope":
        return {"y": st["y"]}
    if kind == "attention":
        return {"out": st["out"]}
    if kind == "commit":       # moved as they are: codes are compared as codes
        codes = lambda x: x.view(torch.int8) if x.element_size() == 1 else x
        return {"k": codes(st["k_cache"]), "v": codes(st["v_cache"]), "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    got = {"k": st["k_out"], "v": st["v_out"]}
    return dict(got, q=st["q_out"]) if kind == "append" else got


def run(st):
    case = st["case"]
    kind = case["kind"]
    if own:
        _run_own(st)
    elif kind == "rope":
        st["y"].copy_(_turn(st["x"].float(), st))
    elif kind == "append":
        _plain_append(st)
    elif kind == "read":
        for x in ("k", "v"):
            r = case["rows"]
            st[x + "_out"].copy_(st[x + "_cache"][:, :, :r].float() * st[x + "_scale"][:, :, :r, None])
    elif kind == "attention":
        _plain_attention(st)
    else:
        _plain_commit(st)
    return _outputs(st)


def _run_own(st):
    from paper_2604_16498_amd import binding as F

    case = st["case"]
    kind = case["kind"]
    if "made" not in st:       # the descriptors and the workspace, which a program makes once
        st["made"] = True
        if "increments" in st:
            st["rope"] = F.make_rope_desc(st["increments"], case["style"], st["factor"])
        if "k_cache" in st:
            st["cache"] = F.make_kv_cache(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
        if kind == "attention":
            st["ws"] = F.workspace(F.forge_attn_tree_workspace_bytes(st["cache"], st["q"].shape[2], case["seq"], case["pos"]))
    if kind == "rope":
        F.forge_rope_apply(st["rope"], st["x"], st["y"], st["positions"])
    elif kind == "append":
        F.forge_kv_append(st["cache"], st["k"], st["v"], st["seq_pos"], case["pos"], rope=st["rope"], positions=st["positions"],
                          q=st["q"], q_out=st["q_out"])
        F.forge_kv_read(st["cache"], st["k_out"], st["v_out"], seq_pos=st["seq_pos"], max_pos=case["pos"])
    elif kind == "read":
        F.forge_kv_read(st["cache"], st["k_out"], st["v_out"])
    elif kind == "attention":
        F.forge_attn_tree(st["cache"], st["q"], st["out"], st["seq_pos"], case["pos"], visible=st["visible"], workspace=st["ws"])
    else:
        F.forge_kv_commit(st["cache"], st["path"], st["taken"], st["seq_pos"], case["pos"])


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits


def work(case):
    hq, hkv, dh, _, _ = SHAPES[case["shape"]]
    B, kind = case["batch"], case["kind"]
    store = case.get("store", "same")
    row = dh + 4 if store in TOP else dh * (4 if store == "fp32" else 2)      # a cached row of k or v, its scale with it
    if kind == "read":
        return {"bytes": 2.0 * B * hkv * case["rows"] * (row + 2 * dh), "flops": 2.0 * B * hkv * case["rows"] * dh}
    n = case["seq"]
    if kind == "rope":
        es = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": 2.0 * B * n * (hq + hkv) * dh * es + 4.0 * B * n, "flops": 3.0 * B * n * (hq + hkv) * dh / case["part"]}
    if kind == "append":       # rows in, q and the cached rows out, those read back out again
        return {"bytes": B * n * (2.0 * (hq + 2 * hkv) * dh + 2 * hq * dh + 2 * hkv * (row + 2 * dh) + 4),
                "flops": 3.0 * B * n * (hq + hkv) * dh / case["part"] + 4.0 * B * n * hkv * dh}
    if kind == "commit":       # half of the drafts, read and written
        return {"bytes": 2.0 * case["layers"] * B * 2 * hkv * row * (n / 2), "flops": 0.0}
    es = 4 if store == "fp32" else 2
    rows = sum(_lengths(case))
    return {"bytes": 2.0 * hkv * (rows + B * n) * row + 2.0 * B * n * hq * dh * es + 8.0 * B * n,
            "flops": 4.0 * hq * dh * n * (rows + B * n / 2)}


def _turned64(x, st, theta, factor):
    case = st["case"]
    a = st["positions"].double()[..., None] * torch.tensor(theta, dtype=torch.float64, device="cuda")
    z = torch.polar(torch.full_like(a, factor), a)[:, :, None]
    x, y = x.double(), x.double().clone()
    r = 2 * len(theta)
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["style"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    w = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * z
    y[..., first], y[..., second] = w.real, w.imag
    return y


def _held64(x, store):
    """The values that rows stand for once they are held in the cache's type."""
    if store == "same":
        return x
    top = x.abs().amax(-1, keepdim=True) / TOP[store]
    top = torch.where(top < 2.0 ** -126, torch.ones_like(top), top)
    if store == "int8":
        return torch.round(x / top) * top
    # four significant bits, steps of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2((x / top).abs().clamp_min(2.0 ** -20))).clamp_min(-6.0) - 3.0)
    return torch.round(x / top / step) * step * top


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind in ("rope", "append"):
        theta, factor = _frequencies(case)
    if kind == "rope":
        return {"y": _turned64(st["x"], st, theta, factor)}
    if kind == "append":
        return {"k": _held64(_turned64(st["k"], st, theta, factor).transpose(1, 2), case["store"]),
                "v": _held64(st["v"].double().transpose(1, 2), case["store"]), "q": _turned64(st["q"], st, theta, factor)}
    if kind == "read":
        return {x: st[x + "_cache"][:, :, :case["rows"]].double() * st[x + "_scale"][:, :, :case["rows"], None].double() for x in ("k", "v")}
    if kind == "commit":
        got = {"k": None, "v": None, "k_scale": None, "v_scale": None}
        for name, key in (("k_cache", "k"), ("v_cache", "v"), ("k_scale", "k_scale"), ("v_scale", "v_scale")):
            x = st[name]
            if x is None or x.element_size() == 1:
                continue
            y = x.double()
            for b, (p, m) in enumerate(zip(st["seq_pos"].tolist(), st["taken"].tolist())):
                y[:, b, :, p:p + m] = x[:, b][:, :, p + st["path"][b, :m].long()].double()
            got[key] = y
        return got
    hkv, dh = st["k_cache"].shape[1], st["k_cache"].shape[3]
    n, hq = st["q"].shape[1:3]
    out = torch.zeros(case["batch"], n, hq, dh, dtype=torch.float64, device="cuda")
    for b, p in enumerate(st["seq_pos"].tolist()):
        bits = st["visible"][b].tolist()
        cut = torch.zeros(n, p + n, dtype=torch.bool, device="cuda")
        cut[:, p:] = torch.tensor([[not v >> j & 1 for j in range(n)] for v in bits], device="cuda")
        for h in range(hkv):
            k, v = (st[x + "_cache"][b, h, :p + n].double() for x in ("k", "v"))
            if st["k_scale"] is not None:
                k, v = k * st["k_scale"][b, h, :p + n, None].double(), v * st["v_scale"][b, h, :p + n, None].double()
            for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                s = (st["q"][b, :, j].double() @ k.T.contiguous() / math.sqrt(dh)).masked_fill(cut, -torch.inf)
                out[b, :, j] = torch.softmax(s, -1) @ v
    return {"out": out.view(case["batch"], n, hq * dh)}
