"""Low-rank adapters of many requests in every kernel and combination of kernels (adapter_plan_cases.py): values against the formula in 64 bits, rows
without an adapter, infinities and NaN in one adapter and in one row, recorded calls."""
import numpy as np
import pytest
import torch

from adapter_plan_cases import CASES
from paper_2604_16498_amd import binding as F
from test_gpu_adapters import ints, runs
from tree_inputs import gpu, normal
from util import host

pytestmark = pytest.mark.gpu
ALL = [(dt, call) for dt in CASES for call, _ in CASES[dt]]
N_ADAPTERS = 5


class Call:
    """x, base [M, ldy], a, b, scale as the library has them (fp64 copies in ref), and the call"""

    def __init__(self, rng, dt, call, positive=False):
        self.M, self.K, self.ends, self.rank, ldy = call
        self.N, self.ldy, self.bf16 = self.ends[-1], ldy or self.ends[-1], dt == "bf16"
        self.dt = torch.bfloat16 if self.bf16 else torch.float32
        draw = lambda *s, std=1.0: np.abs(normal(rng, s, self.bf16, std)) + 0.125 if positive else normal(rng, s, self.bf16, std)
        self.x, self.base = normal(rng, (self.M, self.K), self.bf16), normal(rng, (self.M, self.ldy), self.bf16)
        self.a, self.b = draw(N_ADAPTERS, len(self.ends) * self.rank, self.K, std=self.K ** -0.5), draw(N_ADAPTERS, self.N, self.rank, std=0.5)
        self.scale = rng.uniform(0.5, 2.0, N_ADAPTERS).astype(np.float32)
        self.tx, self.tbase, self.ta, self.tb = (gpu(t, self.dt) for t in (self.x, self.base, self.a, self.b))
        # (as they are in the type: `positive` adds to rounded numbers)
        self.a, self.b = host(self.ta), host(self.tb)
        self.desc = F.make_adapters(self.ta, self.tb, gpu(self.scale), self.ends)
        self.ws = F.workspace(F.forge_adapters_workspace_bytes(self.desc, self.M))

    def run(self, ids, in_place=False, ws=None):
        """-> [M, ldy]; behind it and past its columns everything is as it was"""
        y = torch.full((self.M + 1, self.ldy), 7.0, dtype=self.dt, device="cuda")
        if in_place:
            y[:self.M] = self.tbase
        F.forge_adapters_add(self.desc, self.tx, y[:self.M] if in_place else self.tbase, y[:self.M], ints(ids), workspace=self.ws if ws is None else ws)
        assert (y[self.M] == 7.0).all() and (y[:self.M, self.N:] == (self.tbase[:, self.N:] if in_place else 7.0)).all()
        return y[:self.M]

    def check(self, got, ids):
        ids, got = np.asarray(ids), host(got)[:, :self.N]
        for i in range(N_ADAPTERS):
            rows = np.flatnonzero(ids == i)
            if len(rows) == 0:
                continue
            x, lo, s = self.x[rows].astype(np.float64), 0, float(self.scale[i])
            for p, hi in enumerate(self.ends):
                a, b = self.a[i, p * self.rank:(p + 1) * self.rank].astype(np.float64), self.b[i, lo:hi].astype(np.float64)
                t = x @ a.T
                ref = self.base[rows, lo:hi] + s * (t @ b.T)
                first, second = s * (np.abs(x) @ np.abs(a).T) @ np.abs(b).T, s * np.abs(t) @ np.abs(b).T
                # sums of K and of rank terms in fp32, each of their magnitude; t times scale and, in bf16, its two halves (2^-16); one rounding
                off = first * (self.K + 4) * 2.0 ** -24 + second * ((self.rank + 8) * 2.0 ** -23 + (2.0 ** -16 if self.bf16 else 0.0)) + 2.0 ** -24 * np.abs(ref)
                off = off + (2.0 ** -8 * (np.abs(ref) + off) if self.bf16 else 2.0 ** -24 * np.abs(ref)) + 1e-30
                err = np.abs(got[rows, lo:hi] - ref)
                assert (err <= off).all(), (i, p, float((err / off).max()))
                lo = hi
        none = np.flatnonzero((ids < 0) | (ids >= N_ADAPTERS))
        np.testing.assert_array_equal(got[none], self.base[none, :self.N])


def many_ids(rng, M):
    """requests of any length, tiles and more of ids that are none, and a stretch where every row has another adapter than its neighbour"""
    ids = np.array(runs(rng, M, N_ADAPTERS, max(1, M // 40)))
    ids[M // 5:M // 5 + M // 6] = rng.choice([-1, -2**31, N_ADAPTERS, 2**31 - 1])
    at = slice(M // 2, M // 2 + M // 8)
    ids[at] = np.arange(M)[at] % (N_ADAPTERS + 1) - 1
    ids[-1] = 0                                              # the last row of the last, cut tile counts
    return [int(i) for i in ids]


@pytest.mark.parametrize("dt,call", ALL)
def test_values_and_rows_without_an_adapter(dt, call):
    rng = np.random.default_rng(call[0] + call[3])
    c = Call(rng, dt, call)
    for ids in (many_ids(rng, c.M), [2] * c.M, [-1] * c.M):
        got = c.run(ids)
        c.check(got, ids)
        assert torch.equal(got[:, :c.N], c.run(ids, in_place=True)[:, :c.N])


@pytest.mark.parametrize("dt,call", ALL)
def test_infinities_and_nan_stay_with_their_adapter_and_row(dt, call):
    rng = np.random.default_rng(call[0] + call[3] + 1)
    c = Call(rng, dt, call)
    ids = np.array([(m // 3) % 4 - 1 for m in range(c.M)])                    # -1, 0, 1, 2, three rows each
    clean = c.run(ids)
    c.ta[1, 3, 5] = float("inf")
    c.tb[1, min(33, c.N - 1), 2] = float("nan")
    c.tx[torch.tensor(ids < 0)] = float("nan")               # rows without one
    alone = int(np.flatnonzero(ids == 0)[-1])
    c.tx[alone, 7] = float("nan")
    dirty = c.run(ids)
    rest = torch.tensor((ids != 1) & (np.arange(c.M) != alone), device="cuda")
    assert torch.equal(clean[rest], dirty[rest])
    hit = dirty[torch.tensor(ids == 1, device="cuda")]
    assert torch.isnan(hit[:, min(33, c.N - 1)]).all() and not torch.isfinite(hit[:, :c.ends[0]]).any() and torch.isnan(dirty[alone, :c.N]).all()
    later = [n for n in range(c.ends[0], c.N) if n != min(33, c.N - 1)]       # another part's A
    assert torch.isfinite(hit[:, later]).all()


@pytest.mark.parametrize("dt,call", ALL)
def test_an_infinite_row_stays_infinite(dt, call):
    """positive adapters: an infinite element of x gives its sign everywhere in its row, not NaN, and leaves the other rows alone"""
    rng = np.random.default_rng(call[0] + call[3] + 2)
    c = Call(rng, dt, call, positive=True)
    ids = [m % 2 + 1 for m in range(c.M)]
    clean = c.run(ids)
    up, down = c.M // 2, c.M - 1
    c.tx[up, 1], c.tx[down, c.K - 1] = float("inf"), -float("inf")
    got = c.run(ids)
    assert (got[up, :c.N] == float("inf")).all() and (got[down, :c.N] == -float("inf")).all()
    rest = [m for m in range(c.M) if m not in (up, down)]
    assert torch.equal(got[rest], clean[rest])


@pytest.mark.parametrize("dt", list(CASES))
def test_recorded_calls_of_every_kernel_share_a_workspace(dt):
    """replayed in turn and in the other order, with eager calls on another stream between"""
    rng = np.random.default_rng(5)
    made = [Call(rng, dt, call) for call, _ in CASES[dt]]
    ws = F.workspace(max(c.ws.nbytes for c in made))
    ids = [ints(many_ids(rng, c.M)) for c in made]
    y = [torch.empty_like(c.tbase) for c in made]
    go = lambda i: F.forge_adapters_add(made[i].desc, made[i].tx, made[i].tbase, y[i], ids[i], workspace=ws)
    want, graphs = [], []
    for i in range(len(made)):
        y[i].zero_()
        go(i)
        want.append(y[i].clone())
    for i in range(len(made)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go(i)
        graphs.append(g)
    side = torch.cuda.Stream()
    for turn in range(4):
        for t in y:
            t.zero_()
        for g in graphs[::-1 if turn % 2 else 1]:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(y, want))
        for t in y:
            t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for i in range(len(made)):
                go(i)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(y, want))
    ids[0].fill_(3)                                          # read at replay
    graphs[0].replay()
    torch.cuda.synchronize()
    made[0].check(y[0], [3] * made[0].M)
