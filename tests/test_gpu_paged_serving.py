"""Serving many requests as the operators are used together: pages taken on the device, projections with each request's adapter, rows into pages,
attention over them, requests that come, end and share what is freed.  Against a dense fp64 model of one layer."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from oracle import tree_oracle as T
from paper_2604_16498_amd import binding as F
from tree_inputs import gpu, normal
from util import host

pytestmark = pytest.mark.gpu
D, HQ, HKV, DH, RANK, ADAPTERS, P = 256, 4, 2, 64, 8, 3, 16
NQKV, ENDS, THETA = (HQ + 2 * HKV) * DH, [HQ * DH, (HQ + HKV) * DH, (HQ + 2 * HKV) * DH], T.frequencies(10000.0, DH)[0]


class Model:
    """x -> o = attention(rotated qkv with adapters) . Wo, for packed tokens"""

    def __init__(self, rng, bf16):
        self.bf16, self.dt = bf16, torch.bfloat16 if bf16 else torch.float32
        self.w = {"qkv": normal(rng, (NQKV, D), bf16, D ** -0.5), "o": normal(rng, (D, HQ * DH), bf16, D ** -0.5)}
        self.a = {"qkv": normal(rng, (ADAPTERS, 3 * RANK, D), bf16, D ** -0.5), "o": normal(rng, (ADAPTERS, RANK, HQ * DH), bf16, D ** -0.5)}
        self.b = {"qkv": normal(rng, (ADAPTERS, NQKV, RANK), bf16, 0.3), "o": normal(rng, (ADAPTERS, D, RANK), bf16, 0.3)}
        self.scale = rng.uniform(0.5, 1.5, ADAPTERS).astype(np.float32)
        self.tw = {k: gpu(v, self.dt) for k, v in self.w.items()}
        s = gpu(self.scale)
        self.ad = {k: F.make_adapters(gpu(self.a[k], self.dt), gpu(self.b[k], self.dt), s, ENDS if k == "qkv" else None) for k in self.w}
        inc, factor = F.forge_rope_increments(10000.0, DH)
        self.rope = F.make_rope_desc(inc.cuda(), "half", factor)

    def linear(self, name, x, y, ids, ws):
        F.forge_gemm_bias_gelu(x, self.tw[name], None, None, y, act="none", workspace=ws)
        F.forge_adapters_add(self.ad[name], x, y, y, ids, workspace=ws)

    def workspace(self, M, cache, batch, most):
        sizes = [F.forge_gemm_workspace_bytes(m, n, k, "none", self.dt) for m in range(1, M + 1) for n, k in ((NQKV, D), (D, HQ * DH))]
        sizes += [F.forge_adapters_workspace_bytes(a, M) for a in self.ad.values()]
        return F.workspace(max(sizes + [F.forge_attn_paged_workspace_bytes(cache, HQ, batch, most)]))

    def reference(self, x, adapter):
        """all tokens of one request, x [n, D] -> o [n, D]"""
        n = len(x)
        lin = lambda name, v: O.adapters(v, np.asarray(v, np.float64) @ self.w[name].T.astype(np.float64), self.a[name], self.b[name], self.scale,
                                         [adapter] * n, ENDS if name == "qkv" else [D], RANK)[0]
        qkv = lin("qkv", x).reshape(n, HQ + 2 * HKV, DH)
        turned = T.rotate(qkv[:, :HQ + HKV], np.arange(n)[:, None], THETA, "half")
        out = np.zeros((n, HQ, DH))
        for h in range(HQ):
            k, v = turned[:, HQ + h // (HQ // HKV)], qkv[:, HQ + HKV + h // (HQ // HKV)]
            s = turned[:, h] @ k.T * DH ** -0.5
            s[np.triu_indices(n, 1)] = -np.inf
            p = np.exp(s - s.max(-1, keepdims=True))
            out[:, h] = p @ v / p.sum(-1, keepdims=True)
        return lin("o", out.reshape(n, HQ * DH))


def near(got, want, bf16):
    """fp32: a chain of four products of at most 256 terms, 2e-5.  bf16: an element's rounding is off by at most 2^-8 of it, 2.3e-3 in the
    mean square.  Values, weights, o and the output meet 6 of them: 6^0.5 2.3e-3 = 5.5e-3.  q and k meet 3 each, so that a score, which has the
    size of their elements' product, at most 2.6 with the adapters' share (8 0.3^2 1.5^2 = 1.6 beside 1), is off by 2.6 6^0.5 2.3e-3 = 1.5e-2, and
    a weighted sum by that part of itself: together 1.6e-2 of the whole, and 5 times that where an element is far out."""
    got = host(got)
    err, rms = np.abs(got - want), np.sqrt(np.mean(want ** 2))
    assert (err <= (8e-2 if bf16 else 2e-5) * np.maximum(np.abs(want), rms)).all(), (err / np.maximum(np.abs(want), rms)).max()
    assert not bf16 or np.linalg.norm(err) <= 1.6e-2 * np.linalg.norm(want)


@pytest.mark.parametrize("store", ["fp32", "bf16", "int8"])
def test_requests_come_and_go(store):
    rng = np.random.default_rng(11)
    m = Model(rng, store != "fp32")
    batch, cols, n_pages, most_tokens = 6, 8, 24, 90
    held = {"fp32": torch.float32, "bf16": torch.bfloat16, "int8": torch.int8}[store]
    k, v = (torch.zeros(n_pages, HKV, P, DH, dtype=held, device="cuda") for _ in range(2))
    ks, vs = (torch.ones(n_pages, HKV, P, device="cuda") for _ in range(2)) if store == "int8" else (None, None)
    cache = F.make_paged_cache(k, v, ks, vs)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    free, count, table, lengths = torch.randperm(n_pages, device="cuda").int(), i32(1) + n_pages, i32(batch, cols) - 1, i32(batch)
    pool = F.make_page_pool(free, count, table, P)
    change, granted, starts = i32(batch), i32(batch), i32(batch + 1)
    slots, positions, owners = i32(most_tokens), i32(most_tokens), i32(most_tokens)
    adapter = torch.tensor([0, -1, 2, 1, 0, 2], dtype=torch.int32, device="cuda")
    ws = m.workspace(most_tokens, cache, batch, cols * P)
    said = [np.zeros((0, D), np.float32) for _ in range(batch)]       # the tokens of every request
    assign = lambda: F.forge_pages_assign(pool, lengths, change, lengths, granted, starts, slots, positions, owners)

    def rows(x, T):
        """norm-free layer up to the pages: q [T, HQ, DH] rotated"""
        ids = torch.where(owners[:T] < 0, -1, adapter[owners[:T].clamp_min(0).long()]).int()
        qkv = torch.empty(T, NQKV, dtype=m.dt, device="cuda")
        m.linear("qkv", x, qkv, ids, ws)
        q, kk, vv = (qkv.view(T, -1, DH)[:, a:b] for a, b in ((0, HQ), (HQ, HQ + HKV), (HQ + HKV, HQ + 2 * HKV)))
        F.forge_paged_append(cache, kk, vv, slots[:T], rope=m.rope, positions=positions[:T], q=q, q_out=q)
        return q, ids

    def prompts(new):
        """new tokens of some requests at once; each attends to its own rows, read back from its pages"""
        T = sum(new)
        tokens = [normal(rng, (n, D), m.bf16) for n in new]
        change.copy_(torch.tensor(new, dtype=torch.int32))
        assign()
        assert granted.tolist() == new
        x = gpu(np.concatenate(tokens), m.dt)
        q, ids = rows(x, T)
        o = torch.empty(T, HQ * DH, dtype=m.dt, device="cuda")
        at = 0
        for b, n in enumerate(new):
            if n == 0:
                continue
            said[b] = np.concatenate([said[b], tokens[b]])
            L = len(said[b])
            where = (table[b].repeat_interleave(P) * P + torch.arange(P, device="cuda").repeat(cols))[:L].int()
            kv = [torch.empty(HKV, L, DH, dtype=m.dt, device="cuda") for _ in range(2)]
            F.forge_paged_read(cache, *[t.transpose(0, 1) for t in kv], where)
            aw = F.workspace(F.forge_attn_fused_workspace_bytes(1, HQ, HKV, n, L, DH, m.dt))
            F.forge_attn_fused(q[at:at + n].transpose(0, 1).contiguous()[None], kv[0][None], kv[1][None], o[None, at:at + n], kv_len=L, workspace=aw)
            at += n
        y = torch.empty(T, D, dtype=m.dt, device="cuda")
        m.linear("o", o, y, ids, ws)
        at = 0
        for b, n in enumerate(new):
            if n:
                want = m.reference(said[b], int(adapter[b]))
                if store != "int8":
                    near(y[at:at + n], want[-n:], m.bf16)
                at += n

    # a decode step: one token of every request that runs, recorded once
    x_in, out = torch.zeros(batch, D, dtype=m.dt, device="cuda"), torch.zeros(batch, D, dtype=m.dt, device="cuda")
    o, packed = torch.empty(batch, HQ * DH, dtype=m.dt, device="cuda"), torch.empty(batch, D, dtype=m.dt, device="cuda")
    q_by = torch.empty(batch, HQ, DH, dtype=m.dt, device="cuda")

    def decode():
        torch.clamp(lengths, 0, 1, out=change)
        assign()
        take = owners[:batch].clamp_min(0).long()                      # packed token -> request
        packed.copy_(x_in[take])
        q, ids = rows(packed, batch)
        # (padding tokens of the packed batch carry the first request's values and no slot: they are not put back)
        q_by[torch.where(owners[:batch] >= 0, take, batch - 1)] = q     # the last place is idle here
        F.forge_attn_paged(cache, q_by, o, lengths, table, cols * P, workspace=ws)
        F.forge_gemm_bias_gelu(o, m.tw["o"], None, None, out, act="none", workspace=ws)
        F.forge_adapters_add(m.ad["o"], o, out, out, adapter, workspace=ws)

    prompts([20, 0, 33, 1, 15, 0])
    graph = None
    for step in range(30):
        running = [b for b in range(batch) if len(said[b])]
        new = normal(rng, (batch, D), m.bf16)
        x_in.copy_(gpu(new, m.dt))
        if step == 1:
            keep = [t.clone() for t in (lengths, table, free, count, change, granted, starts, slots, positions, owners)]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                decode()
            for t, w in zip((lengths, table, free, count, change, granted, starts, slots, positions, owners), keep):
                assert torch.equal(t, w)                               # recording runs nothing
        decode() if graph is None else graph.replay()
        torch.cuda.synchronize()
        for b in running:
            said[b] = np.concatenate([said[b], new[b:b + 1]])
            if step % 5 == 0 or step in (1, 29):
                want = m.reference(said[b], int(adapter[b]))[-1:]
                if store != "int8":
                    near(out[b:b + 1], want, m.bf16)
                else:                # rows in int8 move a result by their rounding: 1/254 of a row's largest value, a few percent of the whole
                    assert np.linalg.norm(host(out[b:b + 1]) - want) <= 0.05 * np.linalg.norm(want)
        assert lengths.tolist() == [len(s) for s in said]
        idle = [b for b in range(batch) if not len(said[b])]
        assert (o[idle] == 0).all()
        if step == 8:                    # two requests end, and one comes into what they leave
            change.copy_(torch.tensor([-len(said[0]), 0, 0, -len(said[3]), 0, 0], dtype=torch.int32))
            assign()
            said[0], said[3] = np.zeros((0, D), np.float32), np.zeros((0, D), np.float32)
        if step == 12:
            prompts([5, 40, 0, 0, 2, 0])                               # new ones, and the next turn of a running one
        if step == 20:                   # the last two tokens of a request are taken back
            change.copy_(torch.tensor([0, 0, -2, 0, 0, 0], dtype=torch.int32))
            assign()
            said[2] = said[2][:-2]
    used = sum(-(-len(s) // P) for s in said)
    assert count.tolist() == [n_pages - used]
    there = free[:n_pages - used].tolist() + [p for p in table.flatten().tolist() if p >= 0]
    assert sorted(there) == list(range(n_pages))
