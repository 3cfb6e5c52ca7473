"""Pages of the 4-bit cache: every table, length, count and answer against the bookkeeping done entry after entry, and the
tokens of every sequence read back after it."""
import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import host, i32, starts, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


class Pair:
    """A cache and its model; tokens are numbers that stand for rows of `bank`."""

    def __init__(self, essa, ctx, n_pages, page, max_seqs, max_tokens, layers=2, hkv=2, D=64, seed=0):
        self.essa, self.ctx, self.layers = essa, ctx, layers
        self.kv = essa.KvCache(ctx, layers, hkv, D, n_pages, page, max_seqs, max_tokens)
        self.model = orc.KvPages(n_pages, page, max_seqs, self.kv.max_pages)
        self.g = np.random.default_rng(seed)
        self.bank = [values((4096, hkv, D), self.g, torch.float32) for _ in range(2)]
        self.held = [[orc.kv_values(b[0]).astype(np.float32).astype(np.float64)] for b in self.bank]
        self.next = 0

    def extend(self, seqs, counts):
        new = []
        for c in counts:
            if c < 0:
                new.append(int(c))
            else:
                new.append([(self.next + i) % 4096 for i in range(c)])
                self.next += c
        served = torch.empty(len(seqs), dtype=torch.int32, device="cuda")
        self.essa.essa_kv_extend(self.ctx, self.kv, i32(seqs), i32(counts), served)
        want = self.model.extend(seqs, new)
        assert served.tolist() == want
        rows = [max(c, 0) for c in counts]
        R = sum(rows)
        index = torch.tensor([t for x in new if not isinstance(x, int) for t in x], dtype=torch.long, device="cuda")
        for l in range(self.layers):
            if R:
                self.essa.essa_kv_append(self.ctx, self.kv, l, (self.bank[0][1][index] * (l + 1)), self.bank[1][1][index], self.essa.KvBatch(served, starts(rows), R))
        self.check()
        return want

    def fork(self, src, dst, lens=None):
        served = torch.empty(len(dst), dtype=torch.int32, device="cuda")
        self.essa.essa_kv_fork(self.ctx, self.kv, i32(src), i32(dst), None if lens is None else i32(lens), served)
        want = self.model.fork(src, dst, lens)
        assert served.tolist() == want
        self.check()
        return want

    def free(self, seqs):
        self.essa.essa_kv_free(self.ctx, self.kv, i32(seqs))
        self.model.fork([-1] * len(seqs), seqs)
        self.check()

    def compact(self):
        m, u = torch.empty(len(self.model.refs), dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        self.essa.essa_kv_compact(self.ctx, self.kv, m, u)
        used, where = self.model.compact()
        assert u.item() == used and m.tolist() == where
        self.check()

    def check(self, contents=False):
        assert self.kv.len.tolist() == [len(t) for t in self.model.tokens]
        assert self.kv.refs.tolist() == self.model.refs
        np.testing.assert_array_equal(self.kv.table.cpu().numpy(), self.model.table())
        if not contents:
            return
        lens = [len(t) for t in self.model.tokens]
        R = sum(lens)
        if not R:
            return
        index = np.array([t for x in self.model.tokens for t in x])
        K = torch.empty(R, self.kv.n_kv_heads, self.kv.head_dim, device="cuda")
        V = torch.empty_like(K)
        for l in range(self.layers):
            self.essa.essa_kv_read(self.ctx, self.kv, l, K, V, self.essa.KvBatch(i32(range(len(lens))), starts(lens), R))
            want = orc.kv_values(host(self.bank[0][1] * (l + 1)).astype(np.float32)).astype(np.float32)
            np.testing.assert_array_equal(host(K), want[index].astype(np.float64))
            np.testing.assert_array_equal(host(V), self.held[1][0][index])


@pytest.mark.parametrize("page,n_pages,max_seqs,max_tokens,seed", [(32, 40, 9, 400, 0), (64, 30, 12, 700, 1), (128, 9, 5, 500, 2), (32, 3000, 40, 2000, 3)])
def test_a_random_walk(essa, ctx, page, n_pages, max_seqs, max_tokens, seed):
    p = Pair(essa, ctx, n_pages, page, max_seqs, max_tokens, seed=seed)
    g = np.random.default_rng(100 + seed)
    for turn in range(40):
        n = int(g.integers(1, max_seqs + 1))
        kind = g.choice(["extend", "extend", "fork", "cut", "permute", "free", "compact"])
        print("turn", turn, kind, n, flush=True)
        if kind == "extend":
            p.extend([int(x) for x in g.permutation(max_seqs)[:n]], [int(x) for x in g.integers(0, 3 * page, n)])
        elif kind == "fork":
            p.fork([int(x) for x in g.integers(-1, max_seqs, n)], [int(x) for x in g.permutation(max_seqs)[:n]],
                   None if g.random() < 0.5 else [int(x) for x in g.integers(-1, 4 * page, n)])
        elif kind == "cut":
            s = [int(x) for x in g.permutation(max_seqs)[:n]]
            p.fork(s, s, [int(x) for x in g.integers(0, 3 * page, n)])
        elif kind == "permute":
            p.fork([int(x) for x in g.permutation(max_seqs)], list(range(max_seqs)))
        elif kind == "free":
            p.free([int(x) for x in g.permutation(max_seqs)[:max(1, n // 3)]])
        else:
            p.compact()
        if turn % 4 == 3:
            p.check(contents=True)
    p.compact()
    p.check(contents=True)


def test_entries_that_are_not_served(essa, ctx):
    p = Pair(essa, ctx, 6, 32, 5, 128, layers=1)
    assert p.extend([0, -5, 7, 1, 0], [40, 3, 3, -1, 2]) == [0, -1, -4, -4, -4]
    assert p.extend([1, 2, 3], [129, 128, 10]) == [-3, 2, -2]         # too long; fits; no pages left
    assert p.extend([0, 3, 2], [20, 1, 0]) == [0, -2, 2]              # what needs no page is served behind what found none
    assert p.fork([2, 0], [1, 1]) == [1, -4]
    assert p.fork([0, 2, 9], [3, 3, 0]) == [-2, -4, -4]               # a copy of the partly filled page needs one
    assert p.fork([0], [3], [32]) == [3]                              # a full page does not
    p.check(contents=True)
    p.free([1, -1, 2, 2, 40])
    assert p.fork([0], [2]) == [2]
    p.check(contents=True)


def test_cutting_into_shared_pages(essa, ctx):
    """A cut that leaves a shared page partly filled copies it: the other holder's tokens stay when the first one goes on."""
    p = Pair(essa, ctx, 20, 64, 4, 512)
    p.extend([0], [200])
    p.fork([0, 0], [1, 2])
    p.fork([1], [1], [70])
    p.extend([1], [100])
    p.check(contents=True)
    p.fork([0, 0, 2], [0, 3, 2], [100, 190, 64])                      # cut in place while another entry forks from it
    p.extend([0, 3, 2], [50, 1, 9])
    p.check(contents=True)
    p.fork([0, 1, 2, 3], [1, 2, 3, 0])
    p.check(contents=True)


@pytest.mark.parametrize("max_seqs,n", [(4096, 4096), (1500, 1100)])
def test_many_sequences(essa, ctx, max_seqs, n):
    p = Pair(essa, ctx, 9000, 32, max_seqs, 64, layers=1, hkv=1)
    g = np.random.default_rng(7)
    order = [int(x) for x in g.permutation(max_seqs)[:n]]
    p.extend(order, [int(x) for x in g.integers(0, 65, n)])
    p.free(order[::2])
    p.fork(order[1::2], order[::2][:len(order[1::2])])
    p.compact()
    p.check(contents=True)


def test_on_a_stream_of_its_own(essa):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        p = Pair(essa, ctx, 60, 64, 6, 512)
        p.extend([0, 1], [100, 300])
        p.fork([0, 0, 1, 1], [2, 3, 4, 5])
        p.extend([2, 3, 4, 5], [1, 2, 70, 4])
        p.free([0, 1, 3])
        p.compact()
        p.check(contents=True)
        p.kv.close()
        ctx.close()
