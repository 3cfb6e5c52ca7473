"""A chain of drafted tokens is what causal rows are: the two calls of attention over the 4-bit cache held to one another, without a window, behind one that is wider than the chain,
and, with words that name only the last `window` of a path, behind a narrower one."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
from kv_close import levels, limits
from kv_helpers import Cache, host, i32, starts, values
from kv_masks import tree_words

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 0), (100, 5), (200, 70), (1, 0), (7, 0), (9, 3), (33, 40)])
@pytest.mark.parametrize("many", [1, 14])
def test_a_chain_is_what_causal_rows_are(essa, ctx, dtype, window, sinks, many):
    """Both calls' errors are independent and each within kv_close's limit (fp32 queries: 2^-22 of sum |q k| a score and sqrt(L) 2^-24 of the sums, of which the weights' errors are
    twice), so that their difference is within sqrt 2 of it.  (Their bits differ: a tree's units of work are others, and with them the order of sums.)"""
    lens, rows, hq, D = [120, 64, 300] * many, [9, 64, 33] * many, 4, 128
    c = Cache(essa, ctx, lens, 2, D, 32, dtype=dtype, seed=53)
    R, scale = sum(rows), 1 / math.sqrt(D)
    q, qd = values((R, hq, D), np.random.default_rng(54), dtype, scale=1.5)
    batch, out = essa.KvBatch(i32(range(len(lens))), starts(rows), R), [torch.full((R, hq, D), 5.0, device="cuda") for _ in range(2)]
    trees = [orc.kv_mask(L, n, window, sinks)[:, L - n:] for L, n in zip(lens, rows)]                          # what they see of one another
    essa.essa_kv_attention(ctx, c.kv, 0, qd, out[0], batch, scale, window, sinks=sinks)
    essa.essa_kv_attention(ctx, c.kv, 0, qd, out[1], batch, scale, window, sinks=sinks, tree=tree_words(trees, 1))
    a, y, at = host(out[1]), host(out[0]), 0
    for s, (L, n) in enumerate(zip(lens, rows)):
        seen, g = orc.kv_mask(L, n, window, sinks), hq // 2
        (k, _), (v, size) = levels(c.K[0][s]), levels(c.V[0][s])
        for j in sorted({0, n // 3, n - 1}):
            for h in range(hq):
                diff = a[at + j, h] - y[at + j, h]
                if dtype == torch.bfloat16:
                    _, limit = limits(q[at + j, h].astype(np.float64), k[:, h // g], v[:, h // g], size[:, h // g], seen[j], scale)
                    assert np.sqrt(np.square(diff).mean()) <= math.sqrt(2) * limit, (s, j, h)
                else:
                    _, mass, reach = orc.kv_attention_masked(q[at + j:at + j + 1, h:h + 1].astype(np.float64), k[:, h // g:h // g + 1], v[:, h // g:h // g + 1], seen[j:j + 1], scale)
                    amp = mass[0, 0] + np.abs(v[:, h // g]).max()
                    assert (np.abs(diff) <= math.sqrt(2) * amp * (2.0 ** -21 * reach[0, 0] + math.sqrt(L) * 2.0 ** -24 + 2.0 ** -21)).all(), (s, j, h)
        at += n
    assert (a != 5).any() and np.isfinite(a).all()
    c.kv.close()
