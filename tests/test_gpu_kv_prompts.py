"""Prompts' tiles: every call has one long prompt more, so that it is too much for the kernel that small calls of many rows take."""
import math

import numpy as np
import pytest
import torch

from kv_helpers import Cache, check_attention, host, i32, starts, values

pytestmark = pytest.mark.gpu
LITTLE = 8192                                   # length of a call's row of units (64 columns by 32 tokens, 6 more a unit) up to which it is little


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def _much(hq, hkv):
    """Rows (and tokens) of a prompt that is more than little by itself."""
    return next(n for n in range(256, 20000, 37) if -(-n * hq // hkv // 64) * hkv * (n // 32 + 6) > LITTLE)


def _cache(essa, ctx, lens, hq, hkv, D, page=32, **kw):
    return Cache(essa, ctx, list(lens) + [_much(hq, hkv)], hkv, D, page, dtype=torch.bfloat16, **kw)


def _run(essa, ctx, c, rows, hq, seqs=None, window=0, causal=True, out=torch.bfloat16, scale=None, q_scale=1.5, edit=None, seed=21):
    """The last rows of every sequence; the long prompt's own first and last rows are checked with them."""
    D, long_one, more = c.kv.head_dim, len(c.lens) - 1, c.lens[-1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    seqs = list(range(long_one)) if seqs is None else seqs
    per, R = list(rows) + [more], sum(rows) + more
    q, qd = values((R, hq, D), np.random.default_rng(seed), torch.bfloat16, scale=q_scale)
    if edit is not None:
        edit(q)
        qd = torch.from_numpy(q).cuda().to(torch.bfloat16)
    Y = torch.full((R, hq, D), 5.0, device="cuda", dtype=out)
    print("prompt D=%d heads %d/%d rows=%s window=%d causal=%s" % (D, hq, c.kv.n_kv_heads, per, window, causal), flush=True)
    essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32(seqs + [long_one]), starts(per), R), scale, window, causal)
    y, q = host(Y), q.astype(np.float64)
    n = R - more
    check_attention(y[:n], q[:n], c, seqs, rows, scale, 0, window, causal, out)
    check_attention(y[R - 9:], q[R - 9:], c, [long_one], [9], scale, 0, window, causal, out)
    return y[:n], Y


@pytest.mark.parametrize("D,hq,hkv,page,lens,rows", [
    (128, 14, 2, 64, [513, 700, 64, 33], [513, 300, 64, 1]),
    (64, 6, 6, 32, [300, 1, 130, 65], [300, 1, 129, 65]),
    (128, 3, 1, 1024, [1100, 90], [400, 22]),
    (64, 21, 3, 128, [259, 5, 600], [259, 5, 37]),
    (128, 130, 2, 32, [40, 70], [40, 2]),
    (64, 130, 1, 32, [31, 2, 5], [1, 2, 5]),
])
def test_shapes(essa, ctx, D, hq, hkv, page, lens, rows):
    c = _cache(essa, ctx, lens, hq, hkv, D, page, seed=22)
    _run(essa, ctx, c, rows, hq)
    _run(essa, ctx, c, rows, hq, window=100, out=torch.float32)
    _run(essa, ctx, c, rows, hq, causal=False)


@pytest.mark.parametrize("window", [1, 2, 31, 33, 63, 64, 65, 4000])
def test_windows(essa, ctx, window):
    c = _cache(essa, ctx, [70, 333, 100], 6, 2, 64, 64, seed=23)
    _run(essa, ctx, c, [70, 240, 64], 6, window=window)


def test_rows_that_see_nothing_are_zero(essa, ctx):
    c = _cache(essa, ctx, [50, 0, 3, 200], 8, 2, 128, seed=24)
    y, _ = _run(essa, ctx, c, [200, 2, 70, 90], 8, seqs=[2, -3, 1, 3])
    assert (y[:197] == 0).all() and (y[197:200] != 0).any() and (y[200:272] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
def test_what_is_not_seen_has_no_part(essa, ctx, D):
    lens = [45, 70, 200]

    def edit(K, V, s):
        if s < 3:
            K[5, 0, 3], V[6, 1, D - 2] = np.nan, np.inf
            K[7], V[7] = 3e4, -3e4
            V[-1, 0, 1], K[-1, 1, 0] = np.nan, -np.inf
    c = _cache(essa, ctx, lens, 4, 2, D, 64, seed=25, edit=edit)
    for s, n in enumerate(lens):
        used = -(-n // 64)
        c.kv.pool[int(c.kv.table[s, used - 1])][:, :, -(-(n - 64 * (used - 1)) // 32):] = 255
    c.kv.pool[c.kv.refs == 0] = 255
    _run(essa, ctx, c, [40, 66, 70], 4, window=30)
    y, _ = _run(essa, ctx, c, [40, 66, 70], 4)
    assert np.isnan(y[0]).any()


def test_queries_that_are_not_finite(essa, ctx):
    c = _cache(essa, ctx, [33, 90], 4, 2, 64, seed=26)

    def edit(q):
        q[0, 0, 5], q[30, 3, 63], q[40, 1, 0] = np.inf, -np.inf, np.nan
    y, _ = _run(essa, ctx, c, [33, 80], 4, edit=edit)
    assert np.isnan(y[0, 0]).all() and np.isfinite(y[0, 1:]).all() and np.isnan(y[30, 3]).all() and np.isnan(y[40, 1]).all()


def test_scores_and_values_of_every_size(essa, ctx):
    def rising(K, V, s):
        K *= np.linspace(0.01, 3.0, K.shape[0], dtype=np.float32)[:, None, None]
    for q_scale, v_scale, scale in ((8.0, 1.0, None), (1e-3, 1.0, None), (1e4, 30.0, 1e-5), (1.0, 1000.0, 0.02), (1.0, 1e-2, -0.1), (3.0, 1.0, 0.0)):
        c = _cache(essa, ctx, [300], 4, 2, 128, 64, seed=27, v_scale=v_scale, edit=rising)
        _run(essa, ctx, c, [40], 4, scale=scale, q_scale=q_scale)


def test_the_same_bits_twice_and_on_either_side(essa, ctx):
    """A call that is just little and one that just is not agree within what either may be off by; each repeats itself."""
    hq, hkv, n = 4, 2, 300
    c = _cache(essa, ctx, [n], hq, hkv, 128, seed=28)
    y, a = _run(essa, ctx, c, [n], hq)
    _, b = _run(essa, ctx, c, [n], hq)
    assert torch.equal(a, b)
    q, qd = values((n + c.lens[-1], hq, 128), np.random.default_rng(21), torch.bfloat16, scale=1.5)
    Y = torch.empty(n, hq, 128, device="cuda", dtype=torch.bfloat16)
    essa.essa_kv_attention(ctx, c.kv, 0, qd[:n].contiguous(), Y, essa.KvBatch(i32([0]), starts([n]), n), 1 / math.sqrt(128))
    check_attention(host(Y), q[:n].astype(np.float64), c, [0], [n], 1 / math.sqrt(128))


def test_forked_sequences_share_what_they_read(essa, ctx):
    """Prompts forked whole, cut and copied: their rows over shared pages are those over pages of one's own."""
    c = _cache(essa, ctx, [150], 4, 2, 64, 64, seed=29, spare=8)
    essa.essa_kv_fork(ctx, c.kv, i32([0]), i32([2]), i32([100]))
    assert c.kv.table[2, 0] == c.kv.table[0, 0] and c.kv.table[2, 1] != c.kv.table[0, 1]
    for n, seqs in ((1, [0, 2]), (30, [0, 2])):
        q, qd = values((2 * n, 4, 64), np.random.default_rng(30), torch.bfloat16)
        Y = torch.empty(2 * n, 4, 64, device="cuda")
        essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32(seqs), starts([n, n]), 2 * n), 0.125)
        q, y = q.astype(np.float64), host(Y)
        check_attention(y[:n], q[:n], c, [0], [n], 0.125, out_dtype=torch.float32)
        cut = type("Cut", (), {"K": [[x[:100] for x in c.K[0]]], "V": [[x[:100] for x in c.V[0]]]})
        check_attention(y[n:], q[n:], cut, [0], [n], 0.125, out_dtype=torch.float32)
