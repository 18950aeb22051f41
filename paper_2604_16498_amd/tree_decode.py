"""Generation with drafted trees over a quantised cache: the operators of the drafted-tree section of include/forge.h as a serving
loop uses them.  ``python -m paper_2604_16498_amd.tree_decode`` runs it on a small random model.

A step takes, per sequence, the last token that was chosen (the root) and drafts that may follow it, as a tree.  One pass of the
layers gives the model's choice after every node (`TreeDecoder.verify`).  Walking from the root along drafts that agree with it
finds the accepted branch, whose cache rows are moved together (`TreeDecoder.commit`); the choice after its last node
is the next root.  The tokens are those of one-by-one greedy decoding up to rounding, several a pass where drafts agree: more rows a
pass run other kernels, which add up in another order, so two tokens whose logits are a rounding apart may change places.
"""
from __future__ import annotations

import time
from typing import Dict, List, Optional, Sequence

import torch

from . import binding as F
from . import inputs as I


class TreeDecoder:
    """A decoder stack with a tied token table and rotary positions, its cache in `store` ("int8", "fp8" or "same").

    weights: per layer the tensors of the block descriptor; top: wte [vocab, d], normf_g, normf_b.  drafts: the most nodes of a
    tree, the root among them (at most 64).  scaling: arguments of forge_rope_increments behind the base."""

    def __init__(self, shape: I.BlockShape, weights: Sequence[Dict[str, Optional[torch.Tensor]]], top: Dict[str, Optional[torch.Tensor]],
                 batch: int, cap: int, drafts: int = 16, store: str = "int8", style: str = "half", rot_dim: Optional[int] = None, **scaling):
        if not 1 <= drafts <= 64:
            raise ValueError("a tree has 1 to 64 nodes")
        self.shape, self.top, self.batch, self.cap, self.drafts = shape, top, batch, cap, drafts
        self._weights = weights                                             # (the descriptors hold raw pointers)
        self.layers = [F.make_block_desc(shape, w) for w in weights]
        self.dt = top["wte"].dtype
        rows = (len(weights), batch, shape.kv_heads, cap, shape.head_dim)
        held = {"same": self.dt, "int8": torch.int8, "fp8": torch.float8_e4m3fn}[store]
        k, v = (torch.zeros(rows, dtype=held, device="cuda") for _ in range(2))
        ks, vs = (None, None) if store == "same" else (torch.ones(rows[:-1], device="cuda") for _ in range(2))
        self.cache = F.make_kv_cache(k, v, ks, vs)
        self.rope = None
        if shape.use_rope:
            inc, factor = F.forge_rope_increments(shape.rope_base, rot_dim or shape.head_dim, **scaling)
            self.rope = F.make_rope_desc(inc.cuda(), style, factor)
        self.seq_pos = torch.zeros(batch, dtype=torch.int32, device="cuda")   # cached rows,
        self.held = [0] * batch                                               # and on the host, for bounds
        vocab, d = top["wte"].shape
        self._no_pos = torch.zeros(64, d, dtype=self.dt, device="cuda")       # (positions turn the heads instead)
        self._logits_ld = (vocab + 7) // 8 * 8
        # scratch for any number of nodes and any length: the sizes are not monotone in the nodes
        self._ws = F.workspace(max(F.forge_decoder_block_tree_workspace_bytes(l, self.cache, n, cap - n)
                                   for l in self.layers for n in range(1, 65) if n <= cap))
        self._head_ws = F.workspace(max(F.forge_gemm_workspace_bytes(batch * n, vocab, d, "none", self.dt) for n in range(1, 65)))

    def _pass(self, ids, positions, visible, max_pos):
        """ids [B, n] -> the last layer's rows [B, n, d]; their keys and values are in the cache."""
        if max_pos + ids.shape[1] > self.cap:
            raise ValueError("%d tokens behind %d do not fit the cache of %d" % (ids.shape[1], max_pos, self.cap))
        h = torch.empty(*ids.shape, self.shape.d_model, dtype=self.dt, device="cuda")
        F.forge_embed(ids, self.top["wte"], self._no_pos, h)
        for i, layer in enumerate(self.layers):
            F.forge_decoder_block_tree(layer, self.cache, h, h, self.seq_pos, max_pos, self._ws, rope=self.rope, positions=positions,
                                       visible=visible, layer=i)
        return h

    def _choose(self, h):
        """The greedy token after every row, [B, n] int32."""
        B, n, d = h.shape
        y = torch.empty(B * n, d, dtype=self.dt, device="cuda")
        F.forge_residual_norm(h.view(B * n, d), None, self.top["normf_g"], self.top.get("normf_b"), None, y, eps=self.shape.eps,
                              kind=self.shape.norm)
        vocab = self.top["wte"].shape[0]
        logits = torch.empty(B * n, self._logits_ld, dtype=self.dt, device="cuda")
        F.forge_gemm_bias_gelu(y, self.top["wte"], None, None, logits, act="none", workspace=self._head_ws, n=vocab)
        return logits[:, :vocab].argmax(-1).view(B, n).int()

    def prompt(self, ids: torch.Tensor, lengths: Sequence[int]) -> torch.Tensor:
        """ids [B, S], of sequence b the first lengths[b]; pieces of 64 tokens behind one another.  -> the first chosen tokens [B].
        (What a shorter sequence is padded with is written behind its end, where nothing sees it, and overwritten.)"""
        B, S = ids.shape
        top = max(self.held)
        if B != self.batch or len(lengths) != B or not all(1 <= n <= S for n in lengths) or top + S > self.cap:
            raise ValueError("the prompt does not fit the batch or the cache")
        start = self.seq_pos.clone()
        want = torch.tensor([n - 1 for n in lengths], device="cuda")
        first = torch.empty(B, dtype=torch.int32, device="cuda")
        for s in range(0, S, 64):
            part = ids[:, s:s + 64].contiguous()
            n = part.shape[1]
            chosen = self._choose(self._pass(part, None, None, top + s))
            here = (want >= s) & (want < s + n)
            first = torch.where(here, chosen.gather(1, (want - s).clamp(0, n - 1)[:, None])[:, 0], first)
            self.seq_pos += n
        self.seq_pos = start + torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.held = [h + n for h, n in zip(self.held, lengths)]
        return first

    def verify(self, ids: torch.Tensor, parents: Sequence[Sequence[int]]) -> torch.Tensor:
        """ids [B, n]: node 0 the root, then drafts; parents[b][t] < t the node that draft t follows (of the root -1).  -> the
        model's choice after every node, [B, n]."""
        B, n = ids.shape
        if B != self.batch or len(parents) != B:
            raise ValueError("one tree for each of the %d sequences" % self.batch)
        if n > self.drafts or any(len(p) != n or p[0] != -1 or any(not 0 <= q < t for t, q in enumerate(p) if t) for p in parents):
            raise ValueError("each tree has one root, node 0, and at most %d nodes, parents first" % self.drafts)
        bits, depth = [[0] * n for _ in range(B)], [[0] * n for _ in range(B)]
        for b, tree in enumerate(parents):
            for t, q in enumerate(tree):
                bits[b][t] = (bits[b][q] if t else 0) | 1 << t
                depth[b][t] = depth[b][q] + 1 if t else 0
        signed = torch.tensor([[v - (1 << 64) if v >> 63 else v for v in row] for row in bits], dtype=torch.int64, device="cuda")
        positions = self.seq_pos[:, None] + torch.tensor(depth, dtype=torch.int32, device="cuda")
        return self._choose(self._pass(ids.contiguous(), positions, signed, max(self.held)))

    def commit(self, branches: Sequence[Sequence[int]], n: int) -> None:
        """branches[b]: the accepted nodes of a tree of n, from the root down (none: the cache stays as it was)."""
        if len(branches) != self.batch or not 1 <= n <= min(64, self.cap - max(self.held)):
            raise ValueError("one branch for each of the %d sequences, of a tree that fits the cache" % self.batch)
        if any(not -1 < t < n or (i and t <= p[i - 1]) for p in branches for i, t in enumerate(p)):
            raise ValueError("a branch names nodes of its tree, each behind the one before")
        path = torch.tensor([list(p) + [0] * (n - len(p)) for p in branches], dtype=torch.int32, device="cuda")
        taken = torch.tensor([len(p) for p in branches], dtype=torch.int32, device="cuda")
        F.forge_kv_commit(self.cache, path, taken, self.seq_pos, max(self.held))
        self.seq_pos = self.seq_pos + taken
        self.held = [h + len(p) for h, p in zip(self.held, branches)]


def accepted(ids: List[int], parents: Sequence[int], choices: List[int]) -> List[int]:
    """The nodes from the root along drafts that are what the model chose."""
    path = [0]
    while True:
        nxt = [t for t in range(len(ids)) if parents[t] == path[-1] and ids[t] == choices[path[-1]]]
        if not nxt:
            return path
        path.append(nxt[0])


def generate(model: TreeDecoder, first: torch.Tensor, steps: int, draft) -> List[List[int]]:
    """Tokens per sequence, `first` the roots: `steps` passes.  draft(tokens so far of a sequence) -> (ids, parents) of its tree
    without the root (parent 0: it follows the root); trees of a step have one size, shorter ones are filled up with the root's token
    again, drafts behind the root like any other."""
    out = [[int(t)] for t in first]
    for _ in range(steps):
        trees = [draft(o) for o in out]
        n = 1 + max(len(t[0]) for t in trees)
        ids = [[o[-1]] + list(t[0]) + [o[-1]] * (n - 1 - len(t[0])) for o, t in zip(out, trees)]
        parents = [[-1] + list(t[1]) + [0] * (n - 1 - len(t[1])) for t in trees]
        choices = model.verify(torch.tensor(ids, dtype=torch.int32, device="cuda"), parents).tolist()
        branches = [accepted(i, p, c) for i, p, c in zip(ids, parents, choices)]
        model.commit(branches, n)
        for o, i, c, path in zip(out, ids, choices, branches):
            o.extend(i[t] for t in path[1:])
            o.append(c[path[-1]])
    return out


def random_model(shape: I.BlockShape, layers: int, vocab: int, seed: int = 1):
    """Random weights of a shape, on the GPU: (per-layer tensors, top tensors)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std=0.02: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16).mul_(std)
    d, hd = shape.d_model, shape.q_heads * shape.head_dim
    ws = [{"norm1_g": 1 + normal(d, std=0.1), "norm2_g": 1 + normal(d, std=0.1), "w_qkv": normal(shape.qkv_out, d, std=d ** -0.5),
           "w_o": normal(d, hd, std=hd ** -0.5), "w_up": normal(shape.up_out, d, std=d ** -0.5),
           "w_down": normal(d, shape.d_ff, std=shape.d_ff ** -0.5)} for _ in range(layers)]
    return ws, {"wte": normal(vocab, d, std=1.0), "normf_g": 1 + normal(d, std=0.1), "normf_b": None}


def main():
    shape = I.BlockShape(1024, 16, 4, 64, 2816, norm="rmsnorm", mlp_act="swiglu", use_rope=True, rope_base=500000.0, has_bias=False)
    weights, top = random_model(shape, 8, 32000)
    B, S = 4, 200
    ids = torch.randint(0, 32000, (B, S), device="cuda", dtype=torch.int32)
    lengths = [S, 150, 77, 131]
    scaling = dict(scaling="bands", by=8.0, context=8192.0, low=1.0, high=4.0)
    told: Dict[str, List[List[int]]] = {}
    for name, width, passes in (("one by one", 0, 60), ("trees", 5, 10)):
        model = TreeDecoder(shape, weights, top, B, 1024, store="int8", **scaling)
        first = model.prompt(ids, lengths)
        ref = told.get("one by one")

        def draft(tokens):
            # stands for a small model: what the first run chose in one branch, wrong tokens in another before it
            same = [r for r in ref or [] if r[:len(tokens)] == tokens]
            right = same[0][len(tokens):len(tokens) + width] if same else []
            wrong, n = [(t + 1) % 32000 for t in right], len(right)
            chain = lambda at: [0 if i == 0 else at + i for i in range(n)]
            return wrong + right, chain(0) + chain(n)
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        out = generate(model, first, passes, draft)
        torch.cuda.synchronize()
        told[name] = out
        print("%-10s %3d to %3d tokens a sequence, %.2f ms a pass" % (name, min(map(len, out)), max(map(len, out)),
                                                                      (time.perf_counter() - t0) / passes * 1e3))
    same = [min(len(a), len(b)) for a, b in zip(*told.values())]
    print("agree:", [a[:n] == b[:n] for a, b, n in zip(told["one by one"], told["trees"], same)])


if __name__ == "__main__":
    main()
