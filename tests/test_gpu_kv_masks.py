"""Attention over the 4-bit cache through a window with sinks, and of trees of drafted tokens, against 64 bits."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import Cache, host, i32, starts, values
from kv_masks import ancestors, check_masked, cut, random_tree, tree_words

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


DTYPES = [torch.bfloat16, torch.float32]


def _run(essa, ctx, c, seqs, rows, hq, dtype, window=0, sinks=0, trees=None, words=0, fill=0, layer=0, out=None, seed=11, scale=None, q_scale=1.5, edit=None):
    """trees: [rows, rows] truth values for every entry."""
    D, per = c.kv.head_dim, [1] * len(seqs) if rows is None else rows
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    R = int(sum(per))
    q, qd = values((R, hq, D), np.random.default_rng(seed), dtype, scale=q_scale)
    if edit is not None:
        edit(q)
        qd = torch.from_numpy(q).cuda().to(dtype)
    Y = torch.full((R, hq, D), 5.0, device="cuda", dtype=out or dtype)
    tree = None if trees is None else tree_words(trees, words, fill)
    print("masked D=%d heads %d/%d rows=%s lens=%s window=%d sinks=%d words=%d %s" % (D, hq, c.kv.n_kv_heads, per[:8], c.lens[:8], window, sinks, words, dtype), flush=True)
    essa.essa_kv_attention(ctx, c.kv, layer, qd, Y, essa.KvBatch(i32(seqs), None if rows is None else starts(rows), R), scale, window, sinks=sinks, tree=tree)
    y = host(Y)
    live = [s if 0 <= s < len(c.lens) else -1 for s in seqs]
    masks = [None if s < 0 else orc.kv_mask(c.lens[s], n, window, sinks, None if trees is None else cut(trees[i], words)) for i, (s, n) in enumerate(zip(live, per))]
    check_masked(y, q if dtype == torch.float32 else q.astype(np.float64), c, live, per, scale, masks, layer, Y.dtype, dtype == torch.float32)
    return y, Y


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window,sinks", [(1, 1), (1, 33), (30, 4), (32, 32), (33, 64), (64, 31), (100, 1), (100, 200), (500, 5), (1, 2 ** 31 - 1), (2 ** 31 - 1, 7)])
def test_sinks_of_single_tokens(essa, ctx, dtype, window, sinks):
    lens = [1, 2, 31, 33, 64, 97, 333, 1000, 5]
    c = Cache(essa, ctx, lens, 2, 128, 32, layers=2, dtype=dtype, seed=41)
    _run(essa, ctx, c, [3, 0, -1, 7, 1, 6, 2, 8, 5, 4], None, 6, dtype, window, sinks, layer=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window,sinks", [(1, 2), (20, 40), (64, 3), (33, 100), (200, 64)])
@pytest.mark.parametrize("D,hq,hkv,page", [(128, 10, 2, 64), (64, 6, 3, 32)])
def test_sinks_of_several_rows(essa, ctx, dtype, window, sinks, D, hq, hkv, page):
    lens, rows = [40, 300, 33, 700, 5], [3, 9, 33, 70, 2]
    c = Cache(essa, ctx, lens, hkv, D, page, dtype=dtype, seed=42)
    _run(essa, ctx, c, [0, 1, 2, 3, 4], rows, hq, dtype, window, sinks)


@pytest.mark.parametrize("D,hq,hkv,page,lens,rows,window,sinks", [
    (128, 14, 2, 64, [900, 1500, 64], [900, 300, 64], 100, 4),
    (64, 6, 6, 32, [1300, 1, 130], [1300, 1, 129], 33, 70),
    (128, 3, 1, 1024, [2100, 90], [400, 1], 500, 128),
    (64, 21, 3, 128, [1259, 5, 600], [259, 5, 37], 64, 65),
    (128, 28, 4, 64, [700, 701, 702, 703], [700, 701, 702, 40], 128, 1),
])
def test_sinks_of_prompts(essa, ctx, D, hq, hkv, page, lens, rows, window, sinks):
    """Work enough for the kernel of prompts, and little of it for the other one."""
    many = 3
    c = Cache(essa, ctx, lens * many, hkv, D, page, dtype=torch.bfloat16, seed=43)
    _run(essa, ctx, c, list(range(many * len(lens))), rows * many, hq, torch.bfloat16, window, sinks)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, torch.bfloat16, window, sinks, out=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_sequences_with_sinks(essa, ctx, dtype):
    """The sinks' pages and the window's far from one another in the table; parts of both in different workgroups; twice the same bits."""
    lens = [20011, 7, 9000]
    c = Cache(essa, ctx, lens, 1, 64, 32, dtype=dtype, seed=44)
    for rows in (None, [3, 2, 5], [70, 1, 200]):
        for window, sinks in ((4000, 4000), (300, 5), (9000, 2500)):
            _, a = _run(essa, ctx, c, [0, 1, 2], rows, 7, dtype, window, sinks)
            _, b = _run(essa, ctx, c, [0, 1, 2], rows, 7, dtype, window, sinks)
            assert torch.equal(a, b)


def test_without_sinks_the_bits_are_the_windows(essa, ctx):
    lens, rows = [500, 40, 300], [200, 3, 90]
    c = Cache(essa, ctx, lens, 2, 128, 32, dtype=torch.bfloat16, seed=45)
    q = values((293, 6, 128), np.random.default_rng(46), torch.bfloat16)[1]
    batch = essa.KvBatch(i32([0, 1, 2]), starts(rows), 293)
    out = [torch.empty_like(q) for _ in range(3)]
    essa.essa_kv_attention(ctx, c.kv, 0, q, out[0], batch, 0.1, 50)
    mask = essa.essa._KvMask(50, 0, None, 0)
    import ctypes as C
    assert essa.lib.essa_kv_attention_masked(ctx._h, c.kv._h, 0, q.data_ptr(), 768, 1, 6, batch.ref, 0.1, C.byref(mask), out[1].data_ptr(), 768, 1) == 0
    assert torch.equal(out[0], out[1])
    essa.essa_kv_attention(ctx, c.kv, 0, q, out[0], batch, 0.1)                 # and without a window sinks say nothing
    essa.essa_kv_attention(ctx, c.kv, 0, q, out[2], batch, 0.1, sinks=9)
    assert torch.equal(out[0], out[2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,hq,hkv,page,lens,rows,words", [
    (128, 28, 4, 64, [200, 64, 33, 400], [26, 26, 7, 1], 1),
    (64, 8, 8, 32, [150, 70, 5], [63, 64, 5], 1),
    (128, 5, 1, 128, [300, 129], [65, 128], 2),
    (64, 6, 3, 32, [40, 333, 100, 31], [31, 32, 33, 31], 1),
    (128, 2, 2, 32, [500, 260], [200, 130], 4),
    (64, 4, 1, 64, [90, 90], [70, 70], 1),                     # rows past the words: nobody sees them
    (64, 2, 2, 32, [1100], [1030], 16),
])
def test_trees(essa, ctx, dtype, D, hq, hkv, page, lens, rows, words):
    g = np.random.default_rng(47)
    c = Cache(essa, ctx, lens, hkv, D, page, dtype=dtype, seed=48)
    trees = [ancestors(random_tree(g, n)) for n in rows]
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, dtype, trees=trees, words=words)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, dtype, trees=trees, words=words, fill=1, out=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (10, 33), (50, 0), (100, 70), (1000, 3)])
def test_trees_behind_a_window(essa, ctx, dtype, window, sinks):
    g = np.random.default_rng(49)
    lens, rows = [200, 64, 700, 20], [26, 40, 90, 20]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=dtype, seed=50)
    _run(essa, ctx, c, [0, 1, 2, 3], rows, 6, dtype, window, sinks, [ancestors(random_tree(g, n)) for n in rows], 2)


def test_trees_of_much_work(essa, ctx):
    """Entries that the kernel of prompts takes, of the longest trees, beside single rows; with and without a window."""
    g = np.random.default_rng(51)
    lens = [int(x) for x in g.integers(400, 1100, 36)]
    rows = [1 if i % 9 == 8 else int(g.integers(20, 160)) for i in range(36)]
    c = Cache(essa, ctx, lens, 4, 128, 64, dtype=torch.bfloat16, seed=52)
    trees = [ancestors(random_tree(g, n)) for n in rows]
    _run(essa, ctx, c, list(range(36)), rows, 12, torch.bfloat16, trees=trees, words=3)
    _run(essa, ctx, c, list(range(36)), rows, 12, torch.bfloat16, 200, 9, trees, 3, fill=1, out=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_chain_is_what_causal_rows_are(essa, ctx, dtype):
    """Both calls to the same bounds of the same values.  (Their bits may differ: a tree's units of work are others, and with them the order of sums.)"""
    lens, rows = [120, 64, 300], [9, 64, 33]
    c = Cache(essa, ctx, lens, 2, 128, 32, dtype=dtype, seed=53)
    chains = [np.tril(np.ones((n, n), bool)) for n in rows]
    a, _ = _run(essa, ctx, c, [0, 1, 2], rows, 4, dtype, trees=chains, words=1, out=torch.float32)
    q, qd = values((106, 4, 128), np.random.default_rng(11), dtype, scale=1.5)
    Y = torch.empty(106, 4, 128, device="cuda")
    essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32([0, 1, 2]), starts(rows), 106), 1.0 / math.sqrt(128))
    masks = [orc.kv_mask(length, n) for length, n in zip(lens, rows)]
    check_masked(host(Y), q if dtype == torch.float32 else q.astype(np.float64), c, [0, 1, 2], rows, 1.0 / math.sqrt(128), masks, 0, torch.float32, dtype == torch.float32)
    assert a.shape == tuple(Y.shape)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_see_nothing(essa, ctx, dtype):
    """Skipped entries, empty sequences, rows of a tree without a bit and without a token in front, rows in front of the first token."""
    g = np.random.default_rng(54)
    lens, rows, seqs = [30, 0, 3, 200, 30], [30, 5, 40, 7, 30], [0, 1, 2, 3, -2]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=dtype, seed=55)
    trees = [ancestors(random_tree(g, n)) for n in rows]
    trees[0][3] = trees[0][29] = False
    trees[3][2] = False
    y, _ = _run(essa, ctx, c, seqs, rows, 4, dtype, trees=trees, words=1)
    assert (y[[3, 29]] == 0).all() and (y[30:35] == 0).all() and (y[77] != 0).any()
    _run(essa, ctx, c, seqs, rows, 4, dtype, 3, 2, trees, 1)
    _run(essa, ctx, c, [2, 3], [200, 90], 4, dtype, 20, 4)
    _run(essa, ctx, c, [1, 3, 9], None, 4, dtype, trees=[np.zeros((1, 1), bool), np.ones((1, 1), bool), np.ones((1, 1), bool)], words=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("many", [1, 12])
def test_what_is_not_seen_has_no_part(essa, ctx, dtype, many):
    """NaN, infinities and huge values between the sinks and the window, in rows of the tree that are no ancestors, behind the last token; queries that are not finite."""
    g = np.random.default_rng(56)
    lens, rows = [260, 300] * many, [70, 33] * many

    def edit(K, V, s):
        n = len(K)
        K[9, 0, 3], V[40, 1, 70], V[41, 0, 1] = np.nan, np.inf, -np.nan
        K[50], V[50] = 3e4, -3e4
        V[n - 5, 0, 1], K[n - 20, 1, 0], V[n - 7] = np.nan, -np.inf, np.nan
    c = Cache(essa, ctx, lens, 2, 128, 64, dtype=dtype, seed=57, edit=edit)
    for s, n in enumerate(lens):
        pages = c.kv.table[s].tolist()
        used = -(-n // 64)
        c.kv.pool[pages[used - 1]][:, :, -(-(n - 64 * (used - 1)) // 32):] = 255
    c.kv.pool[c.kv.refs == 0] = 255
    trees = [ancestors(random_tree(g, n, 0.1)) for n in rows]

    def some(q):
        q[3, 1, 5], q[rows[0] + 2, 3, 0] = np.inf, np.nan
    y, _ = _run(essa, ctx, c, list(range(2 * many)), rows, 4, dtype, 100, 8, trees, 2, edit=some)
    assert np.isfinite(y).any() and np.isnan(y).any() and np.isnan(y[3, 1]).all()
    y, _ = _run(essa, ctx, c, list(range(2 * many)), rows, 4, dtype, 30, 8)
    assert np.isfinite(y[0]).all() and np.isnan(y[-1]).any()


@pytest.mark.parametrize("dtype", DTYPES)
def test_row_starts_that_name_rows_twice(essa, ctx, dtype):
    hq, R, entries = 6, 50, 8
    c = Cache(essa, ctx, [100 + i for i in range(entries)], 2, 64, 32, dtype=dtype, seed=58)
    Q, Y = torch.randn(R, hq, 64, device="cuda").to(dtype), torch.full((R + 9, hq, 64), 5.0, device="cuda", dtype=dtype)
    tree = torch.full((R, 1), -1, device="cuda")
    essa.essa_kv_attention(ctx, c.kv, 0, Q, Y[:R], essa.KvBatch(i32(range(entries)), i32([R * (i % 2) for i in range(entries + 1)]), R), 0.1, 20, sinks=3, tree=tree)
    torch.cuda.synchronize()
    assert (Y == 5).all()
    _run(essa, ctx, c, [0, 1], [3, 9], hq, dtype, 20, 3)


@pytest.mark.parametrize("dtype", DTYPES)
def test_spoiled_lengths(essa, ctx, dtype):
    """Lengths past what all pages hold, in a table as wide as tables get."""
    D, pages = 64, 4
    kv = essa.KvCache(ctx, 1, 1, D, pages, page_tokens=32, max_seqs=2, max_tokens=2 ** 31 - 32)
    kv.pool.zero_()
    kv.table.fill_(-1)
    for length in (2 ** 31 - 1, -5, 32 * pages + 1):
        kv.len.fill_(length)
        for rows, batch in ((2, essa.KvBatch(i32([0, 1]))), (140, essa.KvBatch(i32([1, 0]), starts([133, 7]), 140))):
            X, Y = torch.zeros(rows, 1, D, device="cuda", dtype=dtype), torch.full((rows, 1, D), 5.0, device="cuda")
            for window, sinks, tree in ((40, 3, None), (0, 0, torch.full((rows, 16), -1, device="cuda")), (2 ** 31 - 1, 2 ** 31 - 1, torch.full((rows, 3), 0x5555, device="cuda")), (1, 2 ** 31 - 1, None)):
                Y.fill_(5.0)
                essa.essa_kv_attention(ctx, kv, 0, X, Y, batch, 1.0, window, sinks=sinks, tree=tree)
                assert (Y == 0).all()
    kv.close()


def test_recorded(essa):
    """A tree's attention in a recorded step: every replay looks at the masks, lengths and tokens of then."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        g = np.random.default_rng(59)
        lens, rows, hq = [140, 333], [40, 26], 6
        c = Cache(essa, ctx, lens, 2, 128, 32, dtype=torch.bfloat16, seed=60)
        q, qd = values((66, hq, 128), g, torch.bfloat16)
        Y, tree = torch.empty_like(qd), torch.zeros(66, 1, dtype=torch.int64, device="cuda")
        batch = essa.KvBatch(i32([0, 1]), starts(rows), 66)
        call = lambda: essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, batch, 0.1, 90, sinks=5, tree=tree)
        call()
        torch.cuda.synchronize()
        ctx.graph_begin()
        call()
        graph = ctx.graph_end()
        for i in range(4):
            trees = [ancestors(random_tree(g, n)) for n in rows]
            tree.copy_(tree_words(trees, 1))
            now = [n - 7 * i for n in lens]
            c.kv.len[:2] = i32(now)
            Y.fill_(5.0)
            graph.launch()
            torch.cuda.synchronize()
            short = type("Short", (), {"K": [[k[:n] for k, n in zip(c.K[0], now)]], "V": [[v[:n] for v, n in zip(c.V[0], now)]]})
            check_masked(host(Y), q.astype(np.float64), short, [0, 1], rows, 0.1, [orc.kv_mask(n, r, 90, 5, t) for n, r, t in zip(now, rows, trees)])
            call()
        graph.close()
        c.kv.close()
        ctx.close()


def test_two_recorded_calls_of_one_context(essa):
    """Attention of a tree and log probabilities, recorded one by one, share the context's scratch: replayed in turn, with calls that are not recorded between."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        g = np.random.default_rng(61)
        c = Cache(essa, ctx, [9000, 700], 2, 128, 64, dtype=torch.bfloat16, seed=62)
        rows, hq = [9, 30], 6
        qd = values((39, hq, 128), g, torch.bfloat16)[1]
        tree, batch = tree_words([ancestors(random_tree(g, n)) for n in rows], 1), essa.KvBatch(i32([0, 1]), starts(rows), 39)
        logits = values((3, 50001), g, torch.bfloat16)[1]
        tokens = torch.from_numpy(g.integers(0, 50001, (3, 2))).int().cuda()
        Y, Z = torch.empty_like(qd), torch.empty_like(qd)
        logp, h, ids, top = torch.empty(3, 2, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, 7, device="cuda", dtype=torch.int32), torch.empty(3, 7, device="cuda")
        calls = [lambda: essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, batch, 0.1, tree=tree),
                 lambda: essa.essa_token_logprobs(ctx, logits, tokens, logp, 1.0, h, ids, top),
                 lambda: essa.essa_kv_attention(ctx, c.kv, 0, qd, Z, batch, 0.1, 4000, sinks=2000)]
        outs = [[Y], [logp, h, ids, top], [Z]]
        for call in calls:
            call()
        torch.cuda.synchronize()
        want = [[o.clone() for o in out] for out in outs]
        assert torch.isfinite(want[0][0]).all() and not torch.equal(want[0][0], want[2][0])
        graphs = []
        for call in calls:
            ctx.graph_begin()
            call()
            graphs.append(ctx.graph_end())
        for turn in range(4):
            for out in outs:
                for o in out:
                    o.fill_(5)
            for i in ((0, 1, 2), (2, 1, 0), (1, 0, 2), (0, 2, 1))[turn]:
                graphs[i].launch()
                if turn & 1:
                    calls[(i + turn) % 3]()
            torch.cuda.synchronize()
            for out, w in zip(outs, want):
                assert all(torch.equal(a, b) for a, b in zip(out, w))
        for graph in graphs:
            graph.close()
        c.kv.close()
        ctx.close()


def test_a_word_a_row(essa, ctx):
    """tree [R] is tree [R, 1]."""
    g = np.random.default_rng(63)
    c = Cache(essa, ctx, [90, 40], 2, 64, 32, dtype=torch.float32, seed=64)
    rows = [20, 11]
    qd = values((31, 4, 64), g, torch.float32)[1]
    tree, batch, out = tree_words([ancestors(random_tree(g, n)) for n in rows], 1), essa.KvBatch(i32([0, 1]), starts(rows), 31), [torch.empty_like(qd) for _ in range(2)]
    essa.essa_kv_attention(ctx, c.kv, 0, qd, out[0], batch, 0.1, tree=tree)
    essa.essa_kv_attention(ctx, c.kv, 0, qd, out[1], batch, 0.1, tree=tree.view(-1))
    assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_scores_of_a_million(essa, ctx, dtype):
    """Exponents up to 2^21 have steps of a quarter; still every row's weights are of one token or a few, and none of them overflows."""
    lens, rows = [900, 300, 40], [300, 9, 30]
    c = Cache(essa, ctx, lens, 2, 128, 64, dtype=dtype, seed=65)
    for per in (rows, [20, 9, 3], None):
        y, _ = _run(essa, ctx, c, [0, 1, 2], per, 4, dtype, 100, 8, q_scale=2e5)
        assert np.isfinite(y).all() and (np.abs(y).max(-1) > 0.1).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 3.0])
def test_scales(essa, ctx, dtype, scale):
    g = np.random.default_rng(66)
    lens, rows = [300, 90, 500, 64], [70, 9, 200, 64]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=dtype, seed=67)
    trees = [ancestors(random_tree(g, n)) for n in rows]
    for many, per in ((4, rows), (2, [5, 3])):
        _run(essa, ctx, c, list(range(many)), per, 8, dtype, 40, 7, [t[:n, :n] for t, n in zip(trees, per)], 4, scale=scale)
        _run(essa, ctx, c, list(range(many)), per, 8, dtype, 40, 7, scale=scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [[3, 9, 1], [200, 150, 300]])
def test_rows_behind_the_last_entry(essa, ctx, dtype, rows):
    """They are nobody's, and stay as they were; so does memory around Y."""
    n, R = sum(rows), sum(rows) + 21
    c = Cache(essa, ctx, [500, 150, 900], 4, 128, 64, dtype=dtype, seed=68)
    Q = torch.randn(R, 28, 128, device="cuda").to(dtype)
    around = torch.full((R + 4, 28 * 128 + 8), 5.0, device="cuda", dtype=dtype)
    Y = around[2:R + 2, 8:]                                    # rows apart, their beginning on 16 bytes
    tree = torch.full((R, 2), -1, device="cuda")
    for kw in ({"sinks": 3}, {"tree": tree}, {"sinks": 70, "tree": tree}):
        around.fill_(5.0)
        essa.essa_kv_attention(ctx, c.kv, 0, Q, Y, essa.KvBatch(i32([0, 1, 2]), starts(rows), R), 0.1, 60, **kw)
        y = around.clone()
        assert torch.isfinite(y).all() and not (y[2:n + 2, 8:] == 5).all(1).any()
        y[2:n + 2, 8:] = 5.0
        assert (y == 5).all()


@pytest.mark.parametrize("seed", range(24))
def test_any_call(essa, ctx, seed):
    """Lengths, rows, heads, pages, windows, sinks and trees as they come."""
    g = np.random.default_rng(1000 + seed)
    hkv, D, dtype = int(g.integers(1, 4)), int(g.choice([64, 128])), DTYPES[seed % 2]
    n, page = int(g.integers(1, 20)), int(g.choice([32, 64, 256]))
    lens = [int(x) for x in np.exp(g.uniform(0, np.log(1500), n))]
    rows = None if seed % 4 == 3 else [int(min(g.integers(0, g.choice([4, 40, 400])), length + 2)) for length in lens]
    window, sinks = int(g.choice([0, g.integers(1, 10), g.integers(1, 900)])), int(g.choice([0, g.integers(1, 10), g.integers(1, 900)]))
    c = Cache(essa, ctx, lens, hkv, D, page, dtype=dtype, seed=seed)
    seqs = [int(x) if g.random() < 0.95 else -1 for x in g.permutation(n)]
    per = [1] * n if rows is None else [rows[s] if s >= 0 else int(g.integers(0, 5)) for s in seqs]
    if sum(per) == 0:
        per[0] = 1
    trees, words = None, 0
    if g.random() < 0.6 or not (window or sinks):
        trees, words = [ancestors(random_tree(g, k)) if k else np.zeros((0, 0), bool) for k in per], int(g.integers(1, 8))
    _run(essa, ctx, c, seqs, None if rows is None else per, hkv * int(g.integers(1, 9)), dtype, window, sinks, trees, words, fill=int(g.integers(0, 2)), out=torch.float32 if g.random() < 0.3 else None)
