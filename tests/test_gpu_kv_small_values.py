"""Attention over the 4-bit cache does not depend on the size of the values: bf16 queries, fp32 outputs, every group of 64
channels held to the rms of its own output.

A weight is rounded to fp16, and once more as it is multiplied by a value's scale: 2^-11 of itself at most each time, and
independently, so that the rms of an output, a sum of such terms of either sign, is off by sqrt(2 / 3) 2^-11 of itself, half of
that more for what the scores are off by (fp16 keys in calls of much work).  2^-10 is twice as much."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import Cache, host, i32, starts, values

pytestmark = pytest.mark.gpu
LIMIT = 2.0 ** -10


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def _check(essa, ctx, c, rows, hq, window=0, checked=None, seed=41):
    """rows None: one row an entry; checked: how many of an entry's last rows are looked at (all)."""
    kv, n = c.kv, len(c.lens)
    D, per = kv.head_dim, [1] * n if rows is None else rows
    R, scale = sum(per), 1 / math.sqrt(kv.head_dim)
    q, qd = values((R, hq, D), np.random.default_rng(seed), torch.bfloat16, scale=1.4)
    Y = torch.full((R, hq, D), 5.0, device="cuda")
    print("small values D=%d heads %d/%d lens=%s rows=%s window=%d" % (D, hq, kv.n_kv_heads, c.lens, rows, window), flush=True)
    essa.essa_kv_attention(ctx, kv, 0, qd, Y, essa.KvBatch(i32(range(n)), None if rows is None else starts(rows), R), scale, window)
    y, at = host(Y), 0
    for s in range(n):
        m = min(per[s], checked or per[s])
        got, qq = y[at + per[s] - m:at + per[s]], q[at + per[s] - m:at + per[s]].astype(np.float64)
        want, _, _ = orc.kv_attention(qq, orc.kv_values(c.K[0][s]), orc.kv_values(c.V[0][s]), m, scale, window)
        for g in range(0, D, 64):
            a, b = got[..., g:g + 64], want[..., g:g + 64]
            err, size = np.sqrt(np.mean((a - b) ** 2)), np.sqrt(np.mean(b ** 2))
            assert err <= LIMIT * size, (s, g, err / size)
        at += per[s]


@pytest.mark.parametrize("v_scale", [1.0, 1e-3, 1e-4, 1e-5, 1000.0])
@pytest.mark.parametrize("D,hq,hkv", [(128, 28, 4), (64, 6, 2)])
def test_values_of_one_size(essa, ctx, D, hq, hkv, v_scale):
    c = Cache(essa, ctx, [400, 2000, 20000], hkv, D, 64, dtype=torch.bfloat16, seed=40, v_scale=v_scale)
    _check(essa, ctx, c, None, hq)
    _check(essa, ctx, c, [3, 8, 2], hq)


@pytest.mark.parametrize("order", ["rising", "falling", "groups", "one token"])
def test_values_of_many_sizes(essa, ctx, order):
    """Sizes that change along the sequence (up to 1000 times within what a row sees), that differ between a head's groups, or one token far above the others."""
    def edit(K, V, s):
        n = V.shape[0]
        if order == "rising":
            V *= np.geomspace(1e-6, 1e-3, n, dtype=np.float32)[:, None, None]
        elif order == "falling":
            V *= np.geomspace(1.0, 1e-3, n, dtype=np.float32)[:, None, None]
        elif order == "groups":
            V[..., :64] *= 1e-5
            V[..., 64:] *= 300.0
        else:
            V *= 1e-4
            V[n // 2] *= 1e4
    c = Cache(essa, ctx, [300, 5000], 2, 128, 32, dtype=torch.bfloat16, seed=42, edit=edit)
    _check(essa, ctx, c, None, 8)
    _check(essa, ctx, c, [40, 17], 8)
    _check(essa, ctx, c, [2, 3], 8, window=100)


def test_large_values_that_are_not_seen(essa, ctx):
    """In front of a window and behind a row lie the largest values that there are, and NaN: small ones that are seen keep their bits."""
    def edit(K, V, s):
        V *= 1e-5
        V[:-70] = np.where(V[:-70] > 0, 32768.0, -32768.0)
        V[3, 0, 5] = np.nan
    c = Cache(essa, ctx, [333, 90, 1000], 2, 64, 64, dtype=torch.bfloat16, seed=43, edit=edit)
    _check(essa, ctx, c, None, 6, window=60)
    _check(essa, ctx, c, [1, 9, 4], 6, window=60)


@pytest.mark.parametrize("v_scale", [1e-3, 1e-5])
def test_prompts(essa, ctx, v_scale):
    """A call of much work: the rows of its prompt, and of the short entries beside it, are no further off."""
    c = Cache(essa, ctx, [2500, 400, 90], 4, 128, 64, dtype=torch.bfloat16, seed=44, v_scale=v_scale)
    _check(essa, ctx, c, [2500, 1, 70], 28, checked=5)
