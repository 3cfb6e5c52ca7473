"""Attention over the 4-bit cache, element by element against 64 bits, with the bounds that its arithmetic gives (kv_helpers)."""
import math

import numpy as np
import pytest
import torch

from kv_helpers import Cache, check_attention, host, i32, starts, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def _run(essa, ctx, cache, seqs, rows, hq, dtype, scale=None, layer=0, window=0, causal=True, out=None, seed=11, q_scale=1.5, edit=None):
    """Queries of the given type through the call, checked; rows None: one row an entry without row_start."""
    D = cache.kv.head_dim
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    per = [1] * len(seqs) if rows is None else rows
    R = int(sum(per))
    q, qd = values((R, hq, D), np.random.default_rng(seed), dtype, scale=q_scale)
    if edit is not None:
        edit(q)
        qd = torch.from_numpy(q).cuda().to(dtype)
    Y = torch.full((R, hq, D), 5.0, device="cuda", dtype=out or dtype)
    print("attention D=%d heads %d/%d seqs=%d rows=%s window=%d causal=%s %s" % (D, hq, cache.kv.n_kv_heads, len(seqs), per[:8], window, causal, dtype), flush=True)
    essa.essa_kv_attention(ctx, cache.kv, layer, qd, Y, essa.KvBatch(i32(seqs), None if rows is None else starts(rows), R), scale, window, causal)
    y = host(Y)
    qh = q if dtype == torch.float32 else q.astype(np.float64)
    check_attention(y, qh, cache, [s if s < len(cache.lens) else -1 for s in seqs], per, scale, layer, window, causal, Y.dtype)
    return y, Y


DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,hq,hkv,page,lens", [
    (128, 28, 4, 64, [1, 2, 31, 32, 33, 65, 400, 1000]),
    (64, 8, 8, 32, [700, 1, 96, 64, 3]),
    (128, 5, 1, 128, [129, 4, 257]),
    (64, 48, 2, 256, [5, 600]),
    (128, 17, 17, 32, [40]),
])
def test_single_tokens(essa, ctx, dtype, D, hq, hkv, page, lens):
    c = Cache(essa, ctx, lens, hkv, D, page, layers=2, dtype=dtype, seed=2)
    _run(essa, ctx, c, list(range(len(lens))), None, hq, dtype, layer=1)
    _run(essa, ctx, c, list(range(len(lens)))[::-1], None, hq, dtype, layer=0, out=torch.float32)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,hq,hkv,lens,rows", [
    (128, 10, 2, [40, 300, 33, 64], [3, 5, 33, 1]),
    (64, 6, 3, [70, 1, 500, 31], [9, 1, 20, 31]),
    (128, 4, 4, [128, 129, 17], [64, 65, 17]),
    (64, 32, 2, [90, 10], [4, 3]),
])
def test_several_rows(essa, ctx, dtype, D, hq, hkv, lens, rows):
    c = Cache(essa, ctx, lens, hkv, D, 32, dtype=dtype, seed=4)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, dtype)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, dtype, causal=False)


@pytest.mark.parametrize("D,hq,hkv,page,lens,rows", [
    (128, 14, 2, 64, [513, 700, 64], [513, 300, 64]),
    (64, 6, 6, 32, [300, 1, 130], [300, 1, 129]),
    (128, 3, 1, 1024, [1100, 90], [400, 1]),
    (64, 21, 3, 128, [259, 5, 600], [259, 5, 37]),
])
def test_prompts(essa, ctx, D, hq, hkv, page, lens, rows):
    c = Cache(essa, ctx, lens, hkv, D, page, dtype=torch.bfloat16, seed=5)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, torch.bfloat16)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, torch.bfloat16, window=100, out=torch.float32)
    _run(essa, ctx, c, list(range(len(lens))), rows, hq, torch.bfloat16, causal=False)


def test_fp32_prompt(essa, ctx):
    c = Cache(essa, ctx, [200, 66], 2, 64, 32, dtype=torch.float32, seed=6)
    _run(essa, ctx, c, [0, 1], [200, 66], 4, torch.float32)
    _run(essa, ctx, c, [1, 0], [50, 120], 4, torch.float32, window=33)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 4000])
def test_windows(essa, ctx, dtype, window):
    lens, rows = [5, 64, 333, 100], [2, 1, 40, 7]
    c = Cache(essa, ctx, lens, 2, 64, 64, dtype=dtype, seed=7)
    _run(essa, ctx, c, [0, 1, 2, 3], rows, 6, dtype, window=window)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_that_see_nothing_are_zero(essa, ctx, dtype):
    """Skipped entries, empty sequences, and rows in front of a sequence's first token."""
    lens = [50, 0, 3, 200]
    c = Cache(essa, ctx, lens, 2, 128, 32, dtype=dtype, seed=8)
    y, _ = _run(essa, ctx, c, [0, -1, 1, 3, 9], None, 8, dtype)
    assert (y[1] == 0).all() and (y[2] == 0).all() and (y[4] == 0).all()
    y, _ = _run(essa, ctx, c, [2, -3, 1, 3], [40, 2, 70, 5], 8, dtype)
    assert (y[:37] == 0).all() and (y[37:40] != 0).any() and (y[40:112] == 0).all()
    y, _ = _run(essa, ctx, c, [2, 3], [200, 90], 8, dtype)
    assert (y[:197] == 0).all()
    c2 = Cache(essa, ctx, [0, 0], 1, 64, 32, dtype=dtype, seed=8)
    y, _ = _run(essa, ctx, c2, [0, 1], [3, 1], 1, dtype, causal=False)
    assert (y == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [None, [3, 2, 70]])
def test_what_is_not_seen_has_no_part(essa, ctx, dtype, rows):
    """NaN and infinities in tokens behind a row, in front of its window, and in the unused rest of a page; huge values there too."""
    lens = [45, 70, 200]

    def edit(K, V, s):
        K[5, 0, 3], V[6, 1, 70] = np.nan, np.inf
        K[7], V[7] = 3e4, -3e4
        if rows:                                              # the last token is behind the rows before it
            V[-1, 0, 1], K[-1, 1, 0] = np.nan, -np.inf
    c = Cache(essa, ctx, lens, 2, 128, 64, dtype=dtype, seed=9, edit=edit)
    # the rest of the last pages and the free pages: every byte 0xff is a NaN scale
    for s, n in enumerate(lens):
        pages = c.kv.table[s].tolist()
        used = -(-n // 64)
        last = c.kv.pool[pages[used - 1]]
        blocks = -(-(n - 64 * (used - 1)) // 32)
        last[:, :, blocks:] = 255
    live = c.kv.refs.cpu().numpy() > 0
    c.kv.pool[torch.from_numpy(~live).cuda()] = 255
    y, _ = _run(essa, ctx, c, [0, 1, 2], rows, 4, dtype, window=30)
    assert rows is not None or np.isfinite(y).all()
    y, _ = _run(essa, ctx, c, [0, 1, 2], rows, 4, dtype)       # seen: NaN in the heads that look
    assert np.isnan(y[0]).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [None, [2, 80, 3]])
def test_queries_that_are_not_finite(essa, ctx, dtype, rows):
    lens = [33, 90, 300]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=dtype, seed=10)

    def edit(q):
        q[0, 0, 5], q[1, 3, 63], q[2, 1, 0] = np.inf, -np.inf, np.nan
    y, _ = _run(essa, ctx, c, [0, 1, 2], rows, 4, dtype, edit=edit)
    assert np.isnan(y[0, 0]).all() and np.isfinite(y[0, 1:]).all() and np.isnan(y[1, 3]).all() and np.isnan(y[2, 1]).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [None, [40, 2]])
def test_scores_and_values_of_every_size(essa, ctx, dtype, rows):
    """Peaked and flat softmaxes, rising scores (the running maximum moves every block), queries and values large and small."""
    lens = [300, 513]

    def rising(K, V, s):
        K *= np.linspace(0.01, 3.0, K.shape[0], dtype=np.float32)[:, None, None]
    for q_scale, v_scale, scale in ((8.0, 1.0, None), (1e-3, 1.0, None), (1e4, 30.0, 1e-5), (1.0, 1000.0, 0.02), (1.0, 1e-2, -0.1), (3.0, 1.0, 0.0)):
        c = Cache(essa, ctx, lens, 2, 128, 64, dtype=dtype, seed=12, v_scale=v_scale, edit=rising)
        _run(essa, ctx, c, [0, 1], rows, 4, dtype, scale=scale, q_scale=q_scale)


@pytest.mark.parametrize("dtype", DTYPES)
def test_long_sequences_are_split_and_joined(essa, ctx, dtype):
    """One sequence of 20000 tokens beside short ones: the work lies along the length; twice the same bits."""
    lens = [20011, 7, 333]
    c = Cache(essa, ctx, lens, 1, 64, 128, dtype=dtype, seed=13)
    for rows in (None, [3, 2, 5], [70, 1, 200]):
        _, a = _run(essa, ctx, c, [0, 1, 2], rows, 7, dtype)
        _, b = _run(essa, ctx, c, [0, 1, 2], rows, 7, dtype)
        assert torch.equal(a, b)


def test_many_sequences(essa, ctx):
    """More entries than a workgroup has threads, in an order of their own, some skipped."""
    g = np.random.default_rng(14)
    lens = [int(x) for x in g.integers(0, 90, 700)]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=torch.bfloat16, seed=14)
    seqs = [int(s) if g.random() < 0.9 else -1 for s in g.permutation(700)]
    _run(essa, ctx, c, seqs, None, 4, torch.bfloat16)
    rows = [int(x) for x in g.integers(0, 4, 700)]
    _run(essa, ctx, c, seqs, rows, 4, torch.bfloat16)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(8, 0), (1, 0), (8, 3)])
def test_queries_and_outputs_at_any_distance(essa, ctx, dtype, pad, shift):
    D, hq, rows = 64, 4, [1, 40, 3]
    c = Cache(essa, ctx, [33, 80, 5], 2, D, 32, dtype=dtype, seed=15)
    R, w = sum(rows), hq * D
    q, qd = values((R, w), np.random.default_rng(16), dtype)
    flat = torch.zeros(R * (w + pad) + shift, device="cuda", dtype=dtype)
    wide = flat[shift:].view(R, w + pad)
    wide[:, :w] = qd
    out = torch.full((R, w + pad + 2), 9.0, device="cuda", dtype=dtype)
    Y = out[:, 2:w + 2]
    for per in (rows, None):
        n = R if per else 3
        essa.essa_kv_attention(ctx, c.kv, 0, wide[:n, :w], Y[:n], essa.KvBatch(i32([0, 1, 2]), None if per is None else starts(per), n), 0.125)
        qh = (q if dtype == torch.float32 else q.astype(np.float64)).reshape(R, hq, D)[:n]
        check_attention(host(Y[:n]).reshape(n, hq, D), qh, c, [0, 1, 2], per or [1, 1, 1], 0.125, out_dtype=dtype)
        assert (host(out)[:, :2] == 9).all() and (host(out)[:, w + 2:] == 9).all()


def test_recorded_step(essa):
    """Extend, append and attention of a decode step in one recorded graph: every replay is the next token, and equals the step
    issued call by call."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        lens, hkv, hq, D, steps = [30, 63, 5], 2, 6, 128, 40
        g = np.random.default_rng(17)
        K = values((steps, 3, hkv, D), g, torch.bfloat16)[1]
        V = values((steps, 3, hkv, D), g, torch.bfloat16)[1]
        Q = values((steps, 3, hq, D), g, torch.bfloat16)[1]
        caches = [Cache(essa, ctx, lens, hkv, D, 32, dtype=torch.bfloat16, spare=9, seed=18) for _ in range(2)]
        seqs, one, served = i32([0, 1, 2]), i32([1, 1, 1]), i32([0, 0, 0])
        k, v, q, y = K[0].clone(), V[0].clone(), Q[0].clone(), torch.empty_like(Q[0])

        def step(kv):
            essa.essa_kv_extend(ctx, kv, seqs, one, served)
            batch = essa.KvBatch(served)
            essa.essa_kv_append(ctx, kv, 0, k, v, batch)
            essa.essa_kv_attention(ctx, kv, 0, q, y, batch, 0.1)
            return batch
        keep = [step(caches[0].kv), step(caches[1].kv)]          # once, unrecorded
        first = y.clone()
        ctx.graph_begin()
        keep.append(step(caches[0].kv))
        graph = ctx.graph_end()
        want = torch.empty_like(y)
        for t in range(1, steps):
            for a, b in ((k, K), (v, V), (q, Q)):
                a.copy_(b[t])
            keep.append(step(caches[1].kv))
            want.copy_(y)
            y.fill_(3.0)
            graph.launch()
            torch.cuda.synchronize()
            assert torch.equal(y, want), t
            assert torch.equal(caches[0].kv.len, caches[1].kv.len) and torch.equal(caches[0].kv.table, caches[1].kv.table)
        assert caches[0].kv.len[:3].tolist() == [x + steps for x in lens] and not torch.equal(first, y)
        graph.close()
        for c in caches:
            c.kv.close()
        ctx.close()
