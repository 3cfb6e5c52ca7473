"""Keeping a path of drafted rows: tables, lengths, counts and answers against the bookkeeping done entry after entry, the tokens of every
sequence read back, and the bytes of everything else as they were."""
import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import Cache, host, i32, starts, values
from kv_masks import ancestors, check_masked, random_tree, tree_words
from test_gpu_kv_pages import Pair

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def _accept(p, seqs, rows, path, keep, plain=False):
    """path[b]: rows[b] numbers, of which the first keep[b] count."""
    R = sum(rows)
    served = torch.empty(len(seqs), dtype=torch.int32, device="cuda")
    path = [(list(q) + [-7] * c)[:c] for q, c in zip(path, rows)]
    flat = [x for q in path for x in q]
    batch = p.essa.KvBatch(i32(seqs)) if plain else p.essa.KvBatch(i32(seqs), starts(rows), R)
    p.essa.essa_kv_accept(p.ctx, p.kv, batch, i32(flat), i32(keep), served)
    want = p.model.accept(seqs, rows, path, keep)
    assert served.tolist() == want, (served.tolist(), want)
    p.check()
    return want


def _walk(g, n):
    """A path from the root of a tree of n rows."""
    parents, at, walk = random_tree(g, n), int(g.integers(-1, n)), []
    while at >= 0:
        walk.append(at)
        at = parents[at]
    return walk[::-1]


@pytest.mark.parametrize("page,D,hkv,layers,seed", [(32, 64, 2, 2, 0), (64, 128, 2, 3, 1), (256, 64, 3, 1, 2), (32, 128, 5, 15, 3)])
def test_drafting_and_keeping(essa, ctx, page, D, hkv, layers, seed):
    """Steps of every kind of path: none of it, all of it, its beginning, rows far apart, paths of more than a block, over several pages."""
    n = 7
    p = Pair(essa, ctx, 300, page, n, 2500, layers=layers, hkv=hkv, D=D, seed=seed)
    g = np.random.default_rng(200 + seed)
    p.extend(list(range(n)), [0, 1, 31, 32, 33, 65, 300])
    for turn in range(8):
        seqs = [int(x) for x in g.permutation(n)]
        rows = [int(x) for x in g.integers(0, [5, 40, 140, 300][turn % 4], n)]
        served = p.extend(seqs, rows)
        assert served == seqs
        path = []
        for c in rows:
            kind = g.integers(0, 5)
            path.append([] if c == 0 or kind == 0 else list(range(c)) if kind == 1 else list(range(int(g.integers(0, c + 1)))) if kind == 2 else
                        sorted(int(x) for x in g.choice(c, int(g.integers(1, c + 1)), replace=False)) if kind == 3 else _walk(g, c))
        print("turn", turn, rows, [len(x) for x in path], flush=True)
        assert _accept(p, seqs, rows, path, [len(x) for x in path]) == seqs
        p.check(contents=True)


def test_single_rows(essa, ctx):
    """Without row starts: every sequence's last token stays or goes."""
    p = Pair(essa, ctx, 40, 32, 6, 200)
    p.extend(list(range(6)), [1, 33, 64, 65, 100, 7])
    assert _accept(p, [0, 1, -1, 3, 4, 5], [1] * 6, [[0], [0], [0], [], [], [0]], [0, 1, 1, 0, 1, 2], plain=True) == [0, 1, -1, 3, -4, -4]
    p.check(contents=True)


def test_entries_that_are_not_served(essa, ctx):
    p = Pair(essa, ctx, 40, 32, 6, 300, layers=1)
    p.extend([0, 1, 2, 3], [70, 40, 100, 9])
    p.fork([2], [4])                                                  # 4 holds the first three pages of 2
    before = p.kv.pool.clone()
    bad = -4
    assert _accept(p, [0, 0, 9, -3, 1, 3], [5, 5, 5, 5, 5, 5], [[1, 3], [1, 3], [0], [0], [2, 2], [0, 5]], [2, 2, 1, 1, 2, 2]) == [0, bad, bad, -1, bad, bad]
    assert _accept(p, [1, 3, 0, 2], [3, 3, 4, 30], [[-1, 2], [1, 0], [0], [1]], [2, 2, -1, 1]) == [bad] * 4
    assert _accept(p, [1, 3], [41, 9], [[0], [2]], [1, 10]) == [bad, bad]
    assert _accept(p, [2, 4, 5], [4, 4, 1], [[1, 2], [3], [0]], [2, 1, 0]) == [2, 4, bad]     # behind the shared pages; an empty sequence has no rows
    p.check(contents=True)
    live = p.kv.refs > 0
    assert torch.equal(p.kv.pool[~live], before[~live])


def test_other_bytes_stay(essa, ctx):
    """Only the blocks that tokens moved into change, and in them only those tokens' values and what lies behind the sequence's end."""
    p = Pair(essa, ctx, 30, 32, 3, 400, layers=2, hkv=2, D=128, seed=5)
    p.extend([0, 1], [70, 50])
    p.extend([0], [90])
    before, table = p.kv.pool.clone(), p.kv.table.clone()
    _accept(p, [0], [90], [[0, 1, 2, 40, 70]], [5])                   # tokens 70, 71, 72 where they were; 73 and 74 are new: one block
    changed = (p.kv.pool != before).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [int(table[0, 2])]
    p.check(contents=True)
    _accept(p, [0, 1], [5, 1], [[0, 1, 2], [0]], [3, 1])              # nothing moves
    after = p.kv.pool.clone()
    p.extend([2], [33])
    held = table[1, :2].long()
    assert torch.equal(after[held], before[held])


def test_row_starts_that_do_not_ascend(essa, ctx):
    p = Pair(essa, ctx, 30, 32, 4, 400, layers=1)
    p.extend([0, 1, 2, 3], [70, 71, 72, 73])
    pool = p.kv.pool.clone()
    served, R = i32([9] * 4), 20
    essa.essa_kv_accept(ctx, p.kv, essa.KvBatch(i32([0, 1, 2, 3]), i32([0, 30, -5, 99, 3]), R), i32(list(range(R))), i32([20, 0, 0, 0]), served)
    assert served.tolist() == [0, 1, 2, 3]
    assert p.kv.len.tolist()[0] == 70 and p.kv.len.tolist()[2] == 52  # entry 0 owns 0 .. 19 and keeps them, 2 loses twenty
    assert p.kv.len.tolist()[1] == 71 and p.kv.len.tolist()[3] == 73
    assert torch.equal(pool, p.kv.pool)


@pytest.mark.parametrize("layers", [1, 40])
def test_spoiled_lengths_and_tables(essa, ctx, layers):
    """Sequences that hold one another's pages: what is answered is one of two things, and the next call of a sound cache is as ever."""
    kv = essa.KvCache(ctx, layers, 2 if layers > 1 else 1, 64, 4, page_tokens=32, max_seqs=2, max_tokens=2 ** 31 - 32)
    kv.pool.zero_()
    for length in (2 ** 31 - 1, -9, 129):
        for entry in (-1, 2 ** 31 - 1, 3):
            kv.table.fill_(entry)
            kv.refs.fill_(1)
            kv.len.fill_(length)
            served = i32([7, 7])
            essa.essa_kv_accept(ctx, kv, essa.KvBatch(i32([0, 1]), starts([100, 20]), 120), i32([3, 50, 99] + [0] * 97 + [1, 19] + [0] * 18), i32([3, 2]), served)
            torch.cuda.synchronize()
            assert all(x in ((-4,) if length < 0 else (-4, i)) for i, x in enumerate(served.tolist()))
    # the counts are where they were: a sound cache again, moved as it should be
    kv.table.fill_(-1)
    kv.refs.zero_()
    kv.len.zero_()
    essa.essa_kv_extend(ctx, kv, i32([0]), i32([100]))
    X = torch.arange(100, device="cuda").float().view(100, 1, 1).expand(100, kv.n_kv_heads, 64).contiguous()
    essa.essa_kv_append(ctx, kv, layers - 1, X, X, essa.KvBatch(i32([0]), starts([100]), 100))
    for path, left in (([1, 3, 4], 93), ([0, 2], 90)):
        c = 10 if left == 93 else 5
        essa.essa_kv_accept(ctx, kv, essa.KvBatch(i32([0]), starts([c]), c), i32(path + [0] * (c - len(path))), i32([len(path)]))
        assert kv.len.tolist() == [left, 0] and (kv.table[0] >= 0).sum().item() == 3
    Y = torch.empty_like(X[:90])
    essa.essa_kv_read(ctx, kv, layers - 1, Y, torch.empty_like(Y), essa.KvBatch(i32([0]), starts([90]), 90))
    assert Y[:, 0, 0].tolist() == list(range(88)) + [88, 91]
    kv.close()


def test_answers_in_place_of_the_sequences(essa, ctx):
    """served is the batch's own list: answers are those of a list apart, every time (names twice behind refused ones among them)."""
    n = 600
    g = np.random.default_rng(9)
    out = []
    names = [int(x) for x in g.integers(-1, 320, n)]
    keep = [int(x) for x in g.integers(-1, 3, n)]
    for turn in range(6):
        p = Pair(essa, ctx, 1500, 32, 300 + n, 128, layers=3, hkv=2)
        p.extend(list(range(300)), [40] * 300)
        seqs, served = i32(names), i32([9] * n)
        batch = essa.KvBatch(seqs, starts([2] * n), 2 * n)
        essa.essa_kv_accept(ctx, p.kv, batch, i32([0, 1] * n), i32(keep), seqs if turn % 2 else served)
        out.append((seqs if turn % 2 else served).tolist())
        want = p.model.accept(names, [2] * n, [[0, 1]] * n, keep)
        assert out[-1] == want
        p.check()
        p.kv.close()


def test_many_sequences(essa, ctx):
    n = 900
    p = Pair(essa, ctx, 5000, 32, n, 128, layers=1, hkv=1)
    g = np.random.default_rng(8)
    order = [int(x) for x in g.permutation(n)]
    p.extend(order, [int(x) for x in g.integers(0, 40, n)])
    rows = [int(x) for x in g.integers(1, 30, n)]
    p.extend(order, rows)
    path = [_walk(g, c) for c in rows]
    _accept(p, order, rows, path, [len(x) for x in path])
    p.check(contents=True)


def test_a_step_of_drafted_tokens(essa):
    """The calls as a step makes them, recorded and replayed beside the same calls one by one: extend, append, the tree's attention, logits of it,
    the most probable tokens, and the path they agree with; then a plain decode step behind it."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        g = np.random.default_rng(61)
        hkv, hq, D, vocab, lens = 2, 6, 64, 700, [30, 64, 131]
        rows = [9, 13, 5]
        n, R = len(rows), sum(rows)
        parents = [random_tree(g, c) for c in rows]
        trees = [ancestors(x) for x in parents]
        words = tree_words(trees, 1)
        head = values((hq * D, vocab), g, torch.float32)[1]
        made = [Cache(essa, ctx, lens, hkv, D, 32, dtype=torch.bfloat16, spare=20, seed=62) for _ in range(2)]
        k, v, q = (values((R, h, D), g, torch.bfloat16)[1] for h in (hkv, hkv, hq))
        first = np.cumsum([0] + rows)
        depth = torch.tensor([int(t.sum()) for tree in trees for t in tree], device="cuda")
        above = torch.tensor([first[b] + p if p >= 0 else -1 for b, x in enumerate(parents) for p in x], device="cuda")
        entry = torch.tensor([b for b, c in enumerate(rows) for _ in range(c)], device="cuda")
        line = torch.zeros(R, R, dtype=torch.bool, device="cuda")
        for b, tree in enumerate(trees):
            line[first[b]:first[b + 1], first[b]:first[b + 1]] = torch.from_numpy(tree).cuda()
        number = torch.arange(R, device="cuda") - torch.from_numpy(first).cuda()[entry]
        seqs, new, served = i32(range(n)), i32(rows), i32([0] * n)
        batch, plain = essa.KvBatch(served, starts(rows), R), essa.KvBatch(served)
        y, logits = torch.empty(R, hq, D, device="cuda"), torch.empty(R, vocab, device="cuda")
        drafted = torch.randint(0, 3, (R,), device="cuda", dtype=torch.int32)
        logp, ids, top = torch.empty(R, device="cuda"), torch.empty(R, 2, device="cuda", dtype=torch.int32), torch.empty(R, 2, device="cuda")
        path, keep, one = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), i32([1] * n)
        y1 = torch.empty(n, hq, D, device="cuda")
        place = torch.arange(R, device="cuda")

        def step(kv):
            essa.essa_kv_extend(ctx, kv, seqs, new, served)
            essa.essa_kv_append(ctx, kv, 0, k, v, batch)
            essa.essa_kv_attention(ctx, kv, 0, q, y, batch, 0.1, 100, sinks=4, tree=words)
            torch.mul(y.view(R, -1)[:, :vocab % 100 + 1].sum(1, keepdim=True), head[0], out=logits)
            essa.essa_token_logprobs(ctx, logits, drafted, logp, 1.0, None, ids, top)
            # a row is right if it and all of its ancestors are; the deepest right one of each sequence ends the path
            right = (drafted + ids[:, 0]) % 3 != 0
            whole = (line & ~right[None, :]).sum(1) == 0
            score = torch.where(whole, depth * R - place, torch.full_like(depth, -1))
            best = torch.full((n,), -1, device="cuda").scatter_reduce_(0, entry, score, "amax")
            end = torch.where(best >= 0, (-best) % R, torch.zeros_like(best))
            on = line[end][entry, place] & (best >= 0)[entry]
            path.zero_()
            at = torch.from_numpy(first).cuda()[entry] + depth - 1
            path.scatter_add_(0, at, torch.where(on, number, torch.zeros_like(number)).int())
            keep.zero_()
            keep.scatter_add_(0, entry, on.int())
            essa.essa_kv_accept(ctx, kv, batch, path, keep, served)
            essa.essa_kv_extend(ctx, kv, served, one)
            essa.essa_kv_append(ctx, kv, 0, k[:n], v[:n], plain)
            essa.essa_kv_attention(ctx, kv, 0, q[:n], y1, plain, 0.1)

        for c in made:                                               # once, unrecorded
            step(c.kv)
        assert torch.equal(made[0].kv.len, made[1].kv.len)
        ctx.synchronize()
        for t in range(5):
            q.copy_(values((R, hq, D), g, torch.bfloat16)[1])
            k.copy_(values((R, hkv, D), g, torch.bfloat16)[1])
            if t == 0:                                               # the first halves of the step are the framework's calls alone: recorded
                def half(kv):
                    essa.essa_kv_extend(ctx, kv, seqs, new, served)
                    essa.essa_kv_append(ctx, kv, 0, k, v, batch)
                    essa.essa_kv_attention(ctx, kv, 0, q, y, batch, 0.1, 100, sinks=4, tree=words)
                    essa.essa_token_logprobs(ctx, logits, drafted, logp, 1.0, None, ids, top)
                    essa.essa_kv_accept(ctx, kv, batch, path, keep, served)
                ctx.graph_begin()
                half(made[0].kv)
                graph = ctx.graph_end()
            logits.copy_(torch.randn(R, vocab, device="cuda"))
            walk = [_walk(g, c) for c in rows]
            path.copy_(i32([x for w, c in zip(walk, rows) for x in (w + [0] * c)[:c]]))
            keep.copy_(i32([len(w) for w in walk]))
            half(made[1].kv)
            want = [x.clone() for x in (y, logp, ids, top, served)]
            for x in (y, logp, top):
                x.fill_(9.0)
            graph.launch()
            torch.cuda.synchronize()
            for a, b in zip(want, (y, logp, ids, top, served)):
                assert torch.equal(a, b), t
            for a, b in ((made[0].kv.len, made[1].kv.len), (made[0].kv.table, made[1].kv.table), (made[0].kv.refs, made[1].kv.refs)):
                assert torch.equal(a, b), t
            for c in made:
                step(c.kv)
        back = []
        for c in made:
            now = c.kv.len[:n].tolist()
            K, V = (torch.empty(sum(now), hkv, D, device="cuda") for _ in range(2))
            essa.essa_kv_read(ctx, c.kv, 0, K, V, essa.KvBatch(seqs, starts(now), sum(now)))
            back.append((K, V))
        assert torch.equal(back[0][0], back[1][0]) and torch.equal(back[0][1], back[1][1]) and torch.isfinite(back[0][0]).all()
        graph.close()
        for c in made:
            c.kv.close()
        ctx.close()


def test_the_rows_that_stay_are_the_trees(essa, ctx):
    """Attention behind an accepted path sees what plain appending of the path's tokens gives: the same bits."""
    g = np.random.default_rng(63)
    hkv, hq, D, base, c = 2, 4, 128, 75, 50
    K, V = (values((base + c, hkv, D), g, torch.bfloat16)[1] for _ in range(2))
    path = [0, 3, 4, 17, 18, 19, 33, 49]
    q = values((2, hq, D), g, torch.bfloat16)[1]
    out = []
    for drafted in (True, False):
        kv = essa.KvCache(ctx, 1, hkv, D, 8, 32, 1, 200)
        kv.pool.fill_(255)
        order = list(range(base)) + ([base + i for i in range(c)] if drafted else [base + i for i in path])
        essa.essa_kv_extend(ctx, kv, i32([0]), i32([len(order)]))
        essa.essa_kv_append(ctx, kv, 0, K[order], V[order], essa.KvBatch(i32([0]), starts([len(order)]), len(order)))
        if drafted:
            essa.essa_kv_accept(ctx, kv, essa.KvBatch(i32([0]), starts([c]), c), i32(path + [0] * (c - len(path))), i32([len(path)]))
        y = torch.empty(2, hq, D, device="cuda")
        essa.essa_kv_attention(ctx, kv, 0, q, y, essa.KvBatch(i32([0]), starts([2]), 2), 0.1)
        out.append((y, kv.len.tolist(), kv.table.tolist(), kv.refs.tolist()))
        kv.close()
    assert torch.equal(out[0][0], out[1][0]) and torch.isfinite(out[0][0]).all() and out[0][1:] == out[1][1:]
