"""Attention over the 4-bit cache with bf16 queries, every row and head held to three times what its roundings are expected to give (kv_close): single tokens,
several rows, prompts on either side of what is little work, windows, sequences that are split and joined, sequences that share pages."""
import math

import numpy as np
import pytest
import torch

from kv_close import check_close
from kv_helpers import Cache, host, i32, starts, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def _check(essa, ctx, c, seqs, rows, hq, window=0, causal=True, most=12, out=torch.float32, scale=None, q_scale=1.5, data=None):
    """rows None: one row an entry.  `most` rows of an entry are looked at, the first and the last among them."""
    D, per = c.kv.head_dim, [1] * len(seqs) if rows is None else rows
    R, scale, g = sum(per), 1 / math.sqrt(D) if scale is None else scale, np.random.default_rng(61)
    q, qd = values((R, hq, D), g, torch.bfloat16, scale=q_scale)
    Y = torch.full((R, hq, D), 5.0, device="cuda", dtype=out)
    essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32(seqs), None if rows is None else starts(rows), R), scale, window, causal)
    y, at, worst = host(Y), 0, 0.0
    for s, n in zip(seqs, per):
        which = sorted({0, n - 1, *(int(x) for x in g.integers(0, n, most - 2))}) if n else []
        src = s if data is None else data[s]
        K, V = (src[0], src[1]) if data is not None else (c.K[0][s], c.V[0][s])
        worst = max(worst, check_close(y[at:at + n], q[at:at + n], K, V, n, scale, window, causal, out == torch.bfloat16, which))
        at += n
    print("D=%d heads %d/%d rows=%s window=%d causal=%s: %.2f of the limit" % (D, hq, c.kv.n_kv_heads, per[:6], window, causal, worst), flush=True)


SHAPES = [(128, 28, 4, 64, [1, 2, 33, 400, 1000]), (64, 8, 8, 32, [700, 3, 64]), (128, 5, 1, 128, [129, 2000]), (64, 48, 2, 256, [5, 600]), (128, 17, 17, 32, [40])]


@pytest.mark.parametrize("D,hq,hkv,page,lens", SHAPES)
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_single_tokens(essa, ctx, D, hq, hkv, page, lens, out):
    c = Cache(essa, ctx, lens, hkv, D, page, dtype=torch.bfloat16, seed=60)
    _check(essa, ctx, c, list(range(len(lens))), None, hq, out=out)


@pytest.mark.parametrize("D,hq,hkv,lens,rows", [(128, 10, 2, [40, 300, 33, 64], [3, 5, 33, 1]), (64, 6, 3, [70, 1, 500, 31], [9, 1, 20, 31]), (128, 4, 4, [128, 1290, 17], [64, 65, 17]), (64, 32, 2, [900, 10], [4, 3])])
def test_several_rows(essa, ctx, D, hq, hkv, lens, rows):
    c = Cache(essa, ctx, lens, hkv, D, 32, dtype=torch.bfloat16, seed=62)
    for window, causal in ((0, True), (0, False), (33, True), (1, True)):
        _check(essa, ctx, c, list(range(len(lens))), rows, hq, window, causal)


@pytest.mark.parametrize("D,hq,hkv,page,lens,rows", [
    (128, 28, 4, 64, [1500, 700, 64], [1500, 300, 64]),
    (64, 6, 6, 32, [2500, 1, 130, 65], [2500, 1, 129, 65]),
    (128, 3, 1, 1024, [5000, 90], [5000, 22]),
    (64, 21, 3, 128, [2000, 5, 600], [1900, 5, 37]),
    (128, 130, 2, 32, [500, 70], [400, 2]),
])
def test_prompts(essa, ctx, D, hq, hkv, page, lens, rows):
    """Calls of much work: rows x heads / 64 units over the blocks of 32 tokens, 6 more a unit, are more than 8192."""
    assert sum(-(-r * hq // hkv // 64) * hkv * (n // 32 + 6) for n, r in zip(lens, rows)) > 8192
    c = Cache(essa, ctx, lens, hkv, D, page, dtype=torch.bfloat16, seed=63)
    for window, causal in ((0, True), (0, False), (100, True)):
        _check(essa, ctx, c, list(range(len(lens))), rows, hq, window, causal)


def test_long_sequences_are_split_and_joined(essa, ctx):
    c = Cache(essa, ctx, [20011, 7, 333], 1, 64, 128, dtype=torch.bfloat16, seed=64)
    for rows in (None, [3, 2, 5], [70, 1, 200]):
        _check(essa, ctx, c, [0, 1, 2], rows, 7, most=6)
    c = Cache(essa, ctx, [50000, 9000], 2, 128, 64, dtype=torch.bfloat16, seed=65)
    for rows in (None, [2, 3], [64, 40]):
        _check(essa, ctx, c, [0, 1], rows, 10, most=4)


@pytest.mark.parametrize("rows", [None, [40, 2]])
def test_scores_and_values_of_every_size(essa, ctx, rows):
    def rising(K, V, s):
        K *= np.linspace(0.01, 3.0, K.shape[0], dtype=np.float32)[:, None, None]
    for q_scale, v_scale, scale in ((8.0, 1.0, None), (1e-3, 1.0, None), (1e4, 30.0, 1e-5), (1.0, 1000.0, 0.02), (1.0, 1e-2, -0.1), (3.0, 1.0, 0.0)):
        c = Cache(essa, ctx, [300, 3000], 2, 128, 64, dtype=torch.bfloat16, seed=66, v_scale=v_scale, edit=rising)
        _check(essa, ctx, c, [0, 1], rows, 4, scale=scale, q_scale=q_scale)


def test_samples_that_share_a_prompt(essa, ctx):
    """Eight samples forked off each of three prompts, each with tokens of its own behind it."""
    lens, hkv, D, own = [150, 333, 64], 4, 128, 9
    c = Cache(essa, ctx, lens, hkv, D, 64, dtype=torch.bfloat16, spare=60, seed=67)
    kv = essa.KvCache(ctx, 1, hkv, D, n_pages=60, page_tokens=64, max_seqs=27, max_tokens=400)
    g, data = np.random.default_rng(68), {}
    for s, n in enumerate(lens):
        essa.essa_kv_extend(ctx, kv, i32([s]), i32([n]))
        essa.essa_kv_append(ctx, kv, 0, *(torch.from_numpy(x[0][s]).cuda().bfloat16() for x in (c.K, c.V)), essa.KvBatch(i32([s]), starts([n]), n))
    samples = list(range(3, 27))
    essa.essa_kv_fork(ctx, kv, i32([i // 8 for i in range(24)]), i32(samples))
    essa.essa_kv_extend(ctx, kv, i32(samples), i32([own] * 24))
    K, Kd = values((24 * own, hkv, D), g, torch.bfloat16, outliers=True)
    V, Vd = values((24 * own, hkv, D), g, torch.bfloat16)
    essa.essa_kv_append(ctx, kv, 0, Kd, Vd, essa.KvBatch(i32(samples), starts([own] * 24), 24 * own))
    for i, s in enumerate(samples):
        data[s] = [np.concatenate([x[0][i // 8], y[own * i:own * (i + 1)]]) for x, y in ((c.K, K), (c.V, V))]
    c.kv.close()
    c.kv = kv
    for rows in (None, [1 + i % 4 for i in range(24)]):
        _check(essa, ctx, c, samples, rows, 28, data=data)
