"""The operators of serving many requests over one pool of cache pages, whose speed is measured beside their plain forms.

A case is a dict of plain values; `listed` gives the fixed ones and `draw` more of the same ranges.  Operators:
  pages      a step's bookkeeping: requests grow and end, pages move between the free stack and their tables, every new token
             gets its slot; then the step taken back, as a scheduler does that drops its last tokens
  append     the new tokens' rows: q and k rotated, k and v into their slots; the rows just written are read back
  read       a history read back from its pages, as a prompt's attention takes it
  attention  one new token per request over its pages
  adapters   the low-rank adapter of each row's request, added to a shared projection's output
Where `own` is false they are computed in elementary torch operations, in 32 bits and rounded once at the end; where it is true
by the calls of paper_2604_16498_amd.binding.
"""
import math
import random

import torch

own = False

# query heads, key / value heads, head size, rotary base, model width of the shapes that this repository serves
SHAPES = {
    "gpt2s": (12, 12, 64, 10000.0, 768),
    "1p3b": (16, 16, 128, 10000.0, 2048),
    "8b": (32, 8, 128, 500000.0, 4096),
}
TOP = {"int8": 127.0, "fp8": 448.0}    # the largest code of a quantised row
PAGES = (16, 32, 64, 128, 256)         # rows of a page


def pages(name, batch, pos, tokens, page, mix, spare=1.5):
    """tokens: the step's new tokens at most.  mix: a prompt, an ended request and idle ones among those that add a token (otherwise all add one).
    spare: free pages over those that the step takes (below 1 some requests are refused)."""
    c = {"kind": "pages", "batch": batch, "pos": pos, "tokens": tokens, "page": page, "mix": mix, "spare": spare}
    return dict(c, name=name) if name else c


def append(name, shape, batch, tokens, pos, page, store, style="half", part=1):
    """tokens: of all requests together; the last twentieth are padding without a slot.  store: "int8", "fp8", "same" (bf16) or "fp32"."""
    c = {"kind": "append", "shape": shape, "batch": batch, "tokens": tokens, "pos": pos, "page": page, "store": store, "style": style,
         "part": part}
    return dict(c, name=name) if name else c


def read(name, shape, rows, page, store):
    """rows: of one request, in the layout of a prompt's attention (heads first)."""
    c = {"kind": "read", "shape": shape, "batch": 1, "rows": rows, "page": page, "store": store}
    return dict(c, name=name) if name else c


def attention(name, shape, batch, rows, page, store):
    """rows: of the longest request, its new one among them; one request in 16 is an idle place of the batch (length 0)."""
    c = {"kind": "attention", "shape": shape, "batch": batch, "rows": rows, "page": page, "store": store}
    return dict(c, name=name) if name else c


def adapters(name, shape, proj, rows, requests, rank, dtype="bf16"):
    """proj: "qkv" (three parts, each with an adapter of its own) or "out".  The rows belong to `requests` requests one after another, each with
    its own adapter, but every fifth without one."""
    c = {"kind": "adapters", "shape": shape, "proj": proj, "rows": rows, "requests": requests, "rank": rank, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the bookkeeping of a decode step of three chats: latency
        pages("pages_b3", 3, 640, 3, 16, False),
        # a serving batch with a prompt coming in, requests ending and idle places
        pages("pages_b256_mixed", 256, 4001, 8192, 16, True),
        # a decode step of three chats with the small model in full precision: latency
        append("append_gpt2s_fp32_b3", "gpt2s", 3, 3, 640, 16, "fp32", style="interleaved", part=4),
        # a prompt beside the tokens of 47 running requests, into int8 pages of the large model
        append("append_8b_int8_t2079", "8b", 48, 2079, 3001, 32, "int8"),
        # the short history of a chat with the small model
        read("read_gpt2s_fp8_r77", "gpt2s", 77, 16, "fp8"),
        # the next turn over a long document: its whole history
        read("read_8b_int8_r30011", "8b", 30011, 64, "int8"),
        # one token of one request of the small model: latency
        attention("attention_gpt2s_b1_r334", "gpt2s", 1, 334, 16, "same"),
        # throughput serving: 64 requests of different lengths
        attention("attention_8b_int8_b64_r2049", "8b", 64, 2049, 16, "int8"),
        # few users with long documents, 16 bits
        attention("attention_8b_b7_r30011", "8b", 7, 30011, 64, "same"),
        # one row of the small model in full precision: latency
        adapters("adapters_gpt2s_fp32_m1_r8", "gpt2s", "out", 1, 1, 8, "fp32"),
        # a decode step of 61 requests, each with its own adapter
        adapters("adapters_8b_qkv_m61_r16", "8b", "qkv", 61, 61, 16),
        # prompts of five requests
        adapters("adapters_8b_out_m4096_r64", "8b", "out", 4096, 5, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["pages", "append", "read", "attention", "attention", "attention", "adapters", "adapters"])
    shape, page = rng.choice(list(SHAPES)), rng.choice(PAGES)
    if kind == "pages":
        batch, mix = _log_int(rng, 1, 256), rng.random() < 0.6
        return pages("", batch, _log_int(rng, 16, 4001), batch + (_log_int(rng, 1, 7900) if mix else 0), page, mix, rng.choice([1.5, 1.5, 0.6]))
    if kind == "adapters":
        fp32 = rng.random() < 0.25
        rows = _log_int(rng, 1, (1024 if fp32 else 4096) // (2 if shape == "8b" else 1))
        return adapters("", shape, rng.choice(["qkv", "out"]), rows, min(rows, _log_int(rng, 1, 64)), 8 * _log_int(rng, 1, 8),
                        "fp32" if fp32 else "bf16")
    store = rng.choice(["int8", "fp8", "same", "fp32"]) if shape == "gpt2s" else rng.choice(["int8", "fp8", "same"])
    if kind == "append":
        tokens = _log_int(rng, 1, 4096)
        return append("", shape, min(tokens, _log_int(rng, 1, 64)), tokens, _log_int(rng, 1, 2001), page, store,
                      rng.choice(["half", "interleaved"]), rng.choice([1, 1, 2, 4]))
    if kind == "read":
        return read("", shape, _log_int(rng, 1, 30011 if shape == "8b" else 15011), page, store)
    batch = _log_int(rng, 1, 64)
    # the rows of all requests together are at most those of the largest listed case
    most = (7 * 20000) // (2 if shape == "1p3b" or store == "fp32" else 1)
    return attention("", shape, batch, _log_int(rng, 1, min(30011, 2 * most // batch)), page, store)


# ---------------------------------------------------------------------------------------------
# inputs


def _up(a, b):
    return -(-a // b)


def _lengths(case):
    """Rows of every request: between a quarter of the longest and all of it; one in 16 has none."""
    b, top = case["batch"], case["rows"]
    return [0 if i % 16 == 5 else top - (3 * top * (b - 1 - i)) // (4 * max(1, b - 1)) for i in range(b)]


def _grown(case, seed):
    """(lengths before a step, their changes)"""
    r = random.Random(seed)
    b, top = case["batch"], case["pos"]
    lens = [r.randint(max(1, top // 4), top) for _ in range(b)]
    change, left = [1] * b, case["tokens"]                                  # (the way back brings no more tokens than the step)
    if case["mix"]:
        for i in range(b):
            k = r.random()
            if k < 0.1:
                lens[i] = change[i] = 0                                      # an idle place
            elif k < 0.2:
                change[i] = -lens[i] if r.random() < 0.7 and lens[i] <= left else -min(left, r.randint(1, min(8, lens[i])))      # ended, or drafts dropped
                left += change[i]
        change[r.randrange(b)] = case["tokens"] - b + 1 if case["tokens"] > b else 1              # a prompt, or its next piece
    return lens, change


def _shares(case):
    """New tokens of every request of an append: one, and the rest a prompt of the last one; padding behind them."""
    t, b = case["tokens"], case["batch"]
    real = t - t // 20
    b = min(b, real)
    return [1] * (b - 1) + [real - b + 1], t - real


def _quantised(x, store):
    """Rows of x as (codes, scales): what an earlier step of the program left in the cache."""
    top = x.float().abs().amax(-1)
    scale = torch.where(top / TOP[store] < 2.0 ** -126, 1.0, top / TOP[store])
    y = x.float() / scale[..., None]
    return (torch.round(y).to(torch.int8) if store == "int8" else y.to(torch.float8_e4m3fn)), scale


def _tables(lens, page, cols, total, r):
    """A table of pages for these lengths (-1: none), the pages in any order; and the free ones."""
    order = list(range(total))
    r.shuffle(order)
    table = []
    for n in lens:
        mine = [order.pop() for _ in range(_up(n, page))]
        table.append(mine + [-1] * (cols - len(mine)))
    return table, order


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = random.Random(seed)
    kind = case["kind"]

    def normal(shape, dt=torch.bfloat16):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)

    def ints(v, dt=torch.int32):
        return torch.tensor(v, dtype=dt, device="cuda")

    def none(*shape, dt=torch.int32):
        return torch.zeros(shape, dtype=dt, device="cuda")

    st = {"case": case}
    if kind == "pages":
        B, P, T = case["batch"], case["page"], case["tokens"]
        lens, change = _grown(case, seed)
        after = [n + c for n, c in zip(lens, change)]
        taken = sum(max(0, _up(a, P) - _up(n, P)) for n, a in zip(lens, after))
        free = int(taken * case["spare"])
        cols = _up(case["pos"] + T, P) + 3
        total = B * (_up(case["pos"], P) + 2) + 2 * _up(T, P)      # (some belong to other batches)
        table, order = _tables(lens, P, cols, total, r)
        order = order[:free]
        st.update(lengths=ints(lens), change=ints(change), table=ints(table), count=ints([len(order)]),
                  free=ints(order + [0] * (total - len(order))))
        for name in ("step", "return"):
            st[name] = {"granted": none(B), "starts": none(B + 1), "slots": none(T), "positions": none(T), "owners": none(T)}
        st["mid"], st["back"] = none(B), none(B)
        return st
    hq, hkv, dh, base, d = SHAPES[case["shape"]]
    if kind == "adapters":
        dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
        n = case["requests"]
        k, cols = d, [hq * dh, (hq + hkv) * dh, (hq + 2 * hkv) * dh] if case["proj"] == "qkv" else [d]
        st["cols"] = cols
        st["x"], st["base"] = normal((case["rows"], k), dt), normal((case["rows"], cols[-1]), dt)
        st["a"] = (normal((n, len(cols) * case["rank"], k), torch.float32) * k ** -0.5).to(dt)
        st["b"] = (normal((n, cols[-1], case["rank"]), torch.float32) * 0.5).to(dt)
        st["scale"] = torch.rand(n, generator=g, device="cuda") + 0.5
        order = list(range(n))
        r.shuffle(order)                       # which adapter a request has
        st["ids"] = ints([-1 if i % 5 == 4 else order[i] for i in (m * n // case["rows"] for m in range(case["rows"]))])
        st["y"] = torch.empty_like(st["base"])
        return st
    P, store = case["page"], case["store"]
    dt = torch.float32 if store == "fp32" else torch.bfloat16
    if kind == "append":
        shares, pad = _shares(case)
        starts = [r.randint(case["pos"] // 4, case["pos"]) for _ in shares]
        lens = [n + s for n, s in zip(starts, shares)]
    else:
        lens = _lengths(case) if kind == "attention" else [case["rows"]]
        r.shuffle(lens)
    cols = _up(max(lens + [case.get("rows", 1)]), P)
    total = sum(_up(n, P) for n in lens) + 5
    table, _ = _tables(lens, P, cols, total, r)
    for name in ("k", "v"):
        x = normal((total, hkv, P, dh), dt)
        st[name + "_pages"], st[name + "_scale"] = _quantised(x, store) if store in TOP else (x, None)
    slot = lambda b, p: table[b][p // P] * P + p % P
    if kind == "append":
        T = case["tokens"]
        where = [(b, n + j) for b, (n, s) in enumerate(zip(starts, shares)) for j in range(s)]
        st["slots"] = ints([slot(b, p) for b, p in where] + [-1] * pad)
        st["positions"] = ints([p for _, p in where] + [0] * pad)
        turn = dh // case["part"]
        st["increments"] = ints([round(base ** (-2.0 * i / turn) / (2 * math.pi) * 2.0 ** 64) for i in range(turn // 2)], torch.int64)
        # q, k and v as the projection leaves them: one row a token, all heads side by side
        rows = normal((T, hq + 2 * hkv, dh), dt)
        st["q"], st["k"], st["v"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        st["q_out"] = none(T, hq, dh, dt=dt)
        st["k_out"], st["v_out"] = none(T, hkv, dh, dt=dt), none(T, hkv, dh, dt=dt)
    elif kind == "read":
        st["slots"] = ints([slot(0, p) for p in range(case["rows"])])
        st["k_out"], st["v_out"] = (none(hkv, case["rows"], dh, dt=dt).transpose(0, 1) for _ in range(2))
    else:
        st["table"], st["lengths"] = ints(table), ints(lens)
        st["q"] = normal((case["batch"], hq, dh), dt)
        st["out"] = none(case["batch"], hq * dh, dt=dt)
    return st


# ---------------------------------------------------------------------------------------------
# the plain forms


def _plain_assign(st, lengths, change, after, out):
    """The table, the free stack and its count move on in place."""
    table, free, count, P = st["table"], st["free"], st["count"], st["case"]["page"]
    B, C = table.shape
    n, c, total, most = lengths.long(), change.long(), free.shape[0], out["slots"].shape[0]
    have = (n + P - 1) // P
    less = torch.where(c <= 0, (n + c).clamp_min(0), n)
    keep = (less + P - 1) // P
    dropped = have - keep
    ends = torch.cumsum(c.clamp_min(0), 0)
    fits = (c > 0) & (n + c <= C * P) & (ends <= most)
    want = torch.where(fits, (n + c + P - 1) // P - have, 0)
    wants = torch.cumsum(want, 0)
    avail = count.long() + dropped.sum()
    ok = fits & ((want == 0) | (wants <= avail))
    want = torch.where(ok, want, 0)
    col = torch.arange(C, device="cuda")
    gone = (col >= keep[:, None]) & (col < have[:, None])
    to = count.long() + (torch.cumsum(dropped, 0) - dropped)[:, None] + col - keep[:, None]
    stack = torch.cat([free, free[:1]]).scatter_(0, torch.where(gone, to, total).flatten(), table.flatten())[:total]
    fresh = (col >= have[:, None]) & (col < (have + want)[:, None])
    at = avail - 1 - ((wants - want)[:, None] + col - have[:, None])
    free.copy_(stack)
    table.copy_(torch.where(fresh, stack[at.clamp(0, total - 1)], torch.where(gone, -1, table)))
    count.copy_(avail - want.sum())
    granted = torch.where(c <= 0, less - n, torch.where(ok, c, 0))
    after.copy_(n + granted)
    out["granted"].copy_(granted)
    out["starts"][1:] = ends.clamp_max(most)
    t = torch.arange(most, device="cuda")
    b = torch.searchsorted(ends, t, right=True)
    real, b = b < B, b.clamp_max(B - 1)
    p = n[b] + t - (ends - c.clamp_min(0))[b]
    slot = table[b, (p // P).clamp(0, C - 1)].long() * P + p % P
    out["slots"].copy_(torch.where(real & ok[b], slot, -1))
    out["positions"].copy_(torch.where(real, p, 0))
    out["owners"].copy_(torch.where(real, b, -1))


def _turn(x, st):
    """x [tokens, heads, dh] in 32 bits, rotated."""
    case = st["case"]
    # positions times increments wrap at whole turns; the rest counts from the nearest quarter
    phase = st["positions"].long()[:, None] * st["increments"]
    quarter = ((phase >> 61) + 1) >> 1
    angle = (phase - (quarter << 62)).float() * (2 * math.pi / 2.0 ** 64)
    c, s = torch.cos(angle), torch.sin(angle)
    odd = (quarter & 1).bool()
    c, s = torch.where(odd, -s, c), torch.where(odd, c, s)
    sign = torch.where((quarter & 2).bool(), -1.0, 1.0)
    c, s = (c * sign)[:, None], (s * sign)[:, None]
    r = x.shape[-1] // case["part"]
    if case["style"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., r:]], -1)


def _plain_read(st, rows):
    """The values of the pages' rows in the slots of the first `rows` tokens."""
    P, slot = st["case"]["page"], st["slots"][:rows].long()
    for name in ("k", "v"):
        x, scale = st[name + "_pages"], st[name + "_scale"]
        got = (x.view(torch.int8) if scale is not None else x)[slot // P, :, slot % P]
        if scale is not None:
            got = got.view(x.dtype).float() * scale[slot // P, :, slot % P][..., None]
        st[name + "_out"][:rows].copy_(got)


def _plain_append(st):
    case = st["case"]
    real = sum(_shares(case)[0])
    P, slot = case["page"], st["slots"][:real].long()
    for name, x in (("k", _turn(st["k"].float(), st)), ("v", st["v"].float())):
        held, scale = st[name + "_pages"], st[name + "_scale"]
        if scale is None:
            held[slot // P, :, slot % P] = x[:real].to(held.dtype)
        else:
            codes, s = _quantised(x[:real], case["store"])
            held.view(torch.int8)[slot // P, :, slot % P] = codes.view(torch.int8)
            scale[slot // P, :, slot % P] = s
    st["q_out"][:real].copy_(_turn(st["q"].float(), st)[:real])
    _plain_read(st, real)


def _plain_attention(st):
    case = st["case"]
    B, hq, dh = st["q"].shape
    P, C, hkv = case["page"], st["table"].shape[1], st["k_pages"].shape[1]
    page = st["table"].long().clamp_min(0)
    seen = torch.arange(C * P, device="cuda") < st["lengths"][:, None]

    def rows(name):
        x, scale = st[name + "_pages"], st[name + "_scale"]
        x = x[page].float() if scale is None else x.view(torch.int8)[page].view(x.dtype).float() * scale[page][..., None]
        return x.transpose(1, 2).reshape(B, hkv, C * P, dh)

    q = st["q"].float().view(B, hkv, hq // hkv, dh)
    s = torch.matmul(q, rows("k").transpose(2, 3).contiguous()) * dh ** -0.5
    s = s.masked_fill(~seen[:, None, None], -torch.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -torch.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, rows("v")) / torch.where(total == 0, 1.0, total)
    st["out"].copy_(o.reshape(B, hq * dh))


def _plain_adapters(st):
    n, rank, cols = st["a"].shape[0], st["case"]["rank"], st["cols"]
    M, parts = st["x"].shape[0], len(cols)
    has = st["ids"] >= 0
    one = torch.zeros(M, n, device="cuda").scatter_(1, st["ids"].long().clamp_min(0)[:, None], (st["scale"][st["ids"].long().clamp_min(0)] * has)[:, None])
    s = torch.matmul(st["x"].float(), st["a"].float().view(-1, st["x"].shape[1]).T).view(M, n, parts, rank)
    s = (s * one[:, :, None, None]).permute(2, 0, 1, 3).reshape(parts * M, n * rank)
    o = torch.matmul(s, st["b"].float().transpose(1, 2).reshape(n * rank, -1)).view(parts, M, -1)
    part = torch.searchsorted(torch.tensor(cols, device="cuda"), torch.arange(cols[-1], device="cuda"), right=True)
    st["y"].copy_(st["base"].float() + o.gather(0, part.expand(1, M, -1))[0])


def _outputs(st):
    kind = st["case"]["kind"]
    if kind == "pages":
        return {"step": st["step"], "back": st["return"], "mid": st["mid"], "after": st["back"], "table": st["table"], "free": st["free"],
                "count": st["count"]}
    if kind == "attention":
        return {"out": st["out"]}
    if kind == "adapters":
        return {"y": st["y"]}
    got = {"k": st["k_out"], "v": st["v_out"]}
    return dict(got, q=st["q_out"]) if kind == "append" else got


def run(st):
    kind = st["case"]["kind"]
    if own:
        _run_own(st)
    elif kind == "pages":
        _plain_assign(st, st["lengths"], st["change"], st["mid"], st["step"])
        _plain_assign(st, st["mid"], -st["step"]["granted"], st["back"], st["return"])
    elif kind == "append":
        _plain_append(st)
    elif kind == "read":
        _plain_read(st, st["case"]["rows"])
    elif kind == "attention":
        _plain_attention(st)
    else:
        _plain_adapters(st)
    return _outputs(st)


def _run_own(st):
    from paper_2604_16498_amd import binding as F

    case = st["case"]
    kind = case["kind"]
    if "made" not in st:       # the descriptors and the workspace, which a program makes once
        st["made"] = True
        if kind == "pages":
            st["pool"] = F.make_page_pool(st["free"], st["count"], st["table"], case["page"])
        elif kind == "adapters":
            st["adapters"] = F.make_adapters(st["a"], st["b"], st["scale"], st["cols"])
            st["ws"] = F.workspace(F.forge_adapters_workspace_bytes(st["adapters"], case["rows"]))
        else:
            st["cache"] = F.make_paged_cache(st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        if kind == "append":
            st["rope"] = F.make_rope_desc(st["increments"], case["style"], 1.0)
        if kind == "attention":
            st["ws"] = F.workspace(F.forge_attn_paged_workspace_bytes(st["cache"], st["q"].shape[1], case["batch"], case["rows"]))
    if kind == "pages":
        F.forge_pages_assign(st["pool"], st["lengths"], st["change"], st["mid"], **st["step"])
        F.forge_pages_assign(st["pool"], st["mid"], -st["step"]["granted"], st["back"], **st["return"])
    elif kind == "append":
        F.forge_paged_append(st["cache"], st["k"], st["v"], st["slots"], rope=st["rope"], positions=st["positions"], q=st["q"], q_out=st["q_out"])
        F.forge_paged_read(st["cache"], st["k_out"], st["v_out"], st["slots"])
    elif kind == "read":
        F.forge_paged_read(st["cache"], st["k_out"], st["v_out"], st["slots"])
    elif kind == "attention":
        F.forge_attn_paged(st["cache"], st["q"], st["out"], st["lengths"], st["table"], case["rows"], workspace=st["ws"])
    else:
        F.forge_adapters_add(st["adapters"], st["x"], st["base"], st["y"], st["ids"], workspace=st["ws"])


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits


def work(case):
    kind = case["kind"]
    if kind == "pages":        # lengths, changes, starts and what was granted; the tokens' slots, positions and owners
        return {"bytes": 2.0 * (4 * 5 * case["batch"] + 4 * 3 * case["tokens"]), "flops": 0.0}
    hq, hkv, dh, _, d = SHAPES[case["shape"]]
    if kind == "adapters":
        es, M, r = 4 if case["dtype"] == "fp32" else 2, case["rows"], case["rank"]
        parts, N = (3, (hq + 2 * hkv) * dh) if case["proj"] == "qkv" else (1, d)
        n = case["requests"] - case["requests"] // 5
        return {"bytes": es * (1.0 * M * d + 2.0 * M * N + n * r * (parts * d + N)) + 4.0 * M, "flops": 2.0 * M * r * (parts * d + N)}
    store = case["store"]
    es = 4 if store == "fp32" else 2
    row = dh + 4 if store in TOP else dh * es      # a cached row of k or v, its scale with it
    if kind == "read":
        return {"bytes": 2.0 * hkv * case["rows"] * (row + es * dh), "flops": 2.0 * hkv * case["rows"] * dh}
    if kind == "append":       # rows in, q and the cached rows out, those read back out again
        T = sum(_shares(case)[0])
        return {"bytes": T * (es * (hq + 2.0 * hkv) * dh + es * hq * dh + 2 * hkv * (2 * row + es * dh) + 12),
                "flops": 3.0 * T * (hq + hkv) * dh / case["part"] + 4.0 * T * hkv * dh}
    rows = sum(_lengths(case))
    return {"bytes": 2.0 * hkv * rows * row + 2.0 * case["batch"] * hq * dh * es, "flops": 4.0 * hq * dh * rows}


def _turned64(x, st):
    case = st["case"]
    _, _, dh, base, _ = SHAPES[case["shape"]]
    r = dh // case["part"]
    theta = torch.tensor([base ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float64, device="cuda")
    a = st["positions"].double()[:, None] * theta
    z = torch.polar(torch.ones_like(a), a)[:, None]
    y = x.double().clone()
    first, second = (slice(0, r // 2), slice(r // 2, r)) if case["style"] == "half" else (slice(0, r, 2), slice(1, r, 2))
    w = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * z
    y[..., first], y[..., second] = w.real, w.imag
    return y


def _held64(x, store):
    """The values that rows stand for once they are held in the cache's type."""
    if store in ("same", "fp32"):
        return x
    top = x.abs().amax(-1, keepdim=True) / TOP[store]
    top = torch.where(top < 2.0 ** -126, torch.ones_like(top), top)
    if store == "int8":
        return torch.round(x / top) * top
    # four significant bits, steps of 2^-9 below 2^-6
    step = torch.exp2(torch.floor(torch.log2((x / top).abs().clamp_min(2.0 ** -20))).clamp_min(-6.0) - 3.0)
    return torch.round(x / top / step) * step * top


def _rows64(st, name, slots):
    """Values of the rows in these slots of all heads, [slots, heads, dh]."""
    P = st["case"]["page"]
    x, scale = st[name + "_pages"], st[name + "_scale"]
    at = (slots // P, slice(None), slots % P)
    if scale is None:
        return x[at].double()
    return x.view(torch.int8)[at].view(x.dtype).double() * scale[at][..., None].double()


def exact(case, seed):
    kind = case["kind"]
    if kind == "pages":        # whole numbers
        return None
    st = prepare(case, seed)
    if kind == "append":
        real = sum(_shares(case)[0])
        got = {"k": _held64(_turned64(st["k"], st), case["store"]), "v": _held64(st["v"].double(), case["store"]), "q": _turned64(st["q"], st)}
        for y in got.values():
            y[real:] = 0
        return got
    if kind == "read":
        return {x: _rows64(st, x, st["slots"].long()) for x in ("k", "v")}
    if kind == "adapters":
        y = st["base"].double()
        for i in set(st["ids"].tolist()) - {-1}:
            mine = (st["ids"] == i).nonzero()[:, 0]
            x, at, lo = st["x"][mine].double(), 0, 0
            for hi in st["cols"]:
                a, b = st["a"][i, at:at + case["rank"]].double(), st["b"][i, lo:hi].double()
                y[mine, lo:hi] += st["scale"][i].double() * ((x @ a.T.contiguous()) @ b.T.contiguous())
                at, lo = at + case["rank"], hi
        return {"y": y}
    P, hkv = case["page"], st["k_pages"].shape[1]
    B, hq, dh = st["q"].shape
    out = torch.zeros(B, hq, dh, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["lengths"].tolist()):
        if n == 0:
            continue
        p = torch.arange(n, device="cuda")
        slots = st["table"][b].long()[p // P] * P + p % P
        k, v = _rows64(st, "k", slots), _rows64(st, "v", slots)
        for h in range(hq):
            g = h // (hq // hkv)
            out[b, h] = torch.softmax(k[:, g].contiguous() @ st["q"][b, h].double() / math.sqrt(dh), 0) @ v[:, g].contiguous()
    return {"out": out.view(B, hq * dh)}
