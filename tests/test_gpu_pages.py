"""The bookkeeping of a paged cache on the GPU against the oracle: whole numbers, equal in every place."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as O
from paper_2604_16498_amd import binding as F

pytestmark = pytest.mark.gpu


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Pool:
    """The same pool twice: on the GPU, and as lists."""

    def __init__(self, rng, n_pages, P, batch, cols, lengths=None):
        order = [int(x) for x in rng.permutation(n_pages)]
        self.P, self.batch, self.lengths = P, batch, list(lengths) if lengths is not None else [0] * batch
        self.table = [[-1] * cols for _ in range(batch)]
        for b, n in enumerate(self.lengths):
            for col in range(-(-n // P)):
                self.table[b][col] = order.pop()
        self.free, self.count = order + [-7] * (n_pages - len(order)), len(order)
        self.t_free, self.t_count, self.t_table, self.t_len = ints(self.free), ints([self.count]), ints(self.table), ints(self.lengths)
        self.desc = F.make_page_pool(self.t_free, self.t_count, self.t_table, P)

    def step(self, change, most, alias=True, guard=5):
        B = self.batch
        out = {n: torch.full((k,), -99, dtype=torch.int32, device="cuda") for n, k in (("granted", B + guard), ("starts", B + 1 + guard),
                                                                                     ("slots", most + guard), ("positions", most + guard),
                                                                                     ("owners", most + guard))}
        after = self.t_len if alias else torch.empty_like(self.t_len)
        cut = {n: t[:t.shape[0] - guard] for n, t in out.items()}
        tokens = [cut[n] for n in ("slots", "positions", "owners")] if most else [None] * 3
        F.forge_pages_assign(self.desc, self.t_len, ints(change), after, cut["granted"], cut["starts"], *tokens)
        self.t_len = after
        got = O.pages_assign(self.free, self.count, self.table, self.P, self.lengths, change, most)
        self.count, self.lengths = got[0], got[1]
        for name, want in zip(("granted", "starts", "slots", "positions", "owners"), got[2:]):
            np.testing.assert_array_equal(out[name].cpu().numpy(), want + [-99] * guard, err_msg=name)
        assert self.t_len.tolist() == self.lengths and self.t_count.tolist() == [self.count]
        np.testing.assert_array_equal(self.t_table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(self.t_free.cpu().numpy(), self.free)
        return got


# batches around a wave, a block's threads and its chunks; tokens around what one launch takes
@pytest.mark.parametrize("batch,most,P", [(1, 1, 16), (1, 300, 16), (3, 256, 32), (64, 256, 16), (64, 257, 16), (65, 100, 64), (256, 256, 16),
                                          (257, 4096, 16), (300, 4097, 32), (1024, 3000, 16), (1025, 6000, 16), (2049, 9000, 1024), (7, 0, 16)])
def test_a_few_steps(batch, most, P):
    rng = np.random.default_rng(batch + most)
    cols = max(2, 2 * most // max(1, batch * P) + 3)
    pool = Pool(rng, batch * (cols + 1) // 2 + 2, P, batch, cols, rng.integers(0, P + 1, batch))
    for step in range(6):
        change = rng.integers(-2 * P, 3, batch)
        change[rng.random(batch) < 0.5] = 1
        change[rng.random(batch) < 0.2] = -10**9                      # ended
        change[int(rng.integers(batch))] = max(1, most // 2)          # a prompt
        if step == 4:
            change = rng.integers(0, 3 * P, batch)                    # more than there is room for
        pool.step([int(c) for c in change], most, alias=bool(step % 2))


def test_who_is_refused():
    """no page, no column, no room among the tokens, and those that need none all the same"""
    rng = np.random.default_rng(3)
    pool = Pool(rng, 8, 16, 6, 3, [16, 10, 16, 0, 47, 5])             # 1 + 1 + 1 + 0 + 3 + 1 pages: one is left
    got = pool.step([1, 3, 20, 1, 2, 1], 64)
    assert got[2] == [1, 3, 0, 0, 0, 1]                                # the page; room in its page; two pages; one page; four columns; room
    pool.step([-17, 0, 40, 33, 1, 0], 50)
    pool.step([2**31 - 1, -2**31, 2**31 - 1, 5, -3, 1], 50)


def test_all_tokens_of_a_full_step_have_rows_of_their_own():
    rng = np.random.default_rng(4)
    pool = Pool(rng, 900, 16, 200, 60, rng.integers(0, 40, 200))
    got = pool.step([int(x) for x in rng.integers(0, 60, 200)], 8000)
    slots = [s for s in got[4] if s >= 0]
    assert len(slots) == len(set(slots)) > 3000


def test_bad_entries_stay_inside():
    """lengths past the table, pages that are none, a count past the stack"""
    rng = np.random.default_rng(5)
    pool = Pool(rng, 40, 16, 4, 4, [20, 3, 40, 0])
    for b, col, v in ((0, 1, -1), (2, 0, 10**6), (2, 2, -5)):
        pool.table[b][col] = v
        pool.t_table[b, col] = v
    pool.lengths = [20, 3, 40, -8]
    pool.t_len.copy_(ints(pool.lengths))
    pool.count = 10**6
    pool.t_count.fill_(10**6)
    pool.step([3, 1, -12, 1], 16)
    pool.lengths = [10**9, 3, 10, 5]
    pool.t_len.copy_(ints(pool.lengths))
    pool.step([-60, 1, 1, 1], 16)


def test_another_stream_and_a_graph():
    rng = np.random.default_rng(6)
    B, most = 20, 64
    a, b = (Pool(np.random.default_rng(6), 200, 16, B, 12, rng_l) for rng_l in [[int(x) for x in rng.integers(1, 60, B)]] * 2)
    change = torch.ones(B, dtype=torch.int32, device="cuda")
    out = lambda: {"granted": torch.empty_like(change), "starts": torch.empty(B + 1, dtype=torch.int32, device="cuda"),
                   **{n: torch.empty(most, dtype=torch.int32, device="cuda") for n in ("slots", "positions", "owners")}}
    oa, ob = out(), out()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        F.forge_pages_assign(b.desc, b.t_len, change, b.t_len, **ob)
    for step in range(30):                       # past several page boundaries
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            F.forge_pages_assign(a.desc, a.t_len, change, a.t_len, **oa)
        side.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(oa[n], ob[n]) for n in oa) and torch.equal(a.t_table, b.t_table) and torch.equal(a.t_len, b.t_len)
        assert torch.equal(a.t_count, b.t_count)
    assert a.t_len.tolist() == [n + 30 for n in a.lengths]
