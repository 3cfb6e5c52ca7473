"""Windows wider than any sequence are no windows, up to the largest number that there is, beside entries with more rows than tokens."""
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


def _call(essa, ctx, c, rows, hq, dtype, window):
    D, R = c.kv.head_dim, sum(rows)
    q, qd = values((R, hq, D), np.random.default_rng(51), dtype)
    Y = torch.full((R, hq, D), 5.0, device="cuda")
    print("window", window, "rows", rows, dtype, flush=True)
    essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32(range(len(rows))), starts(rows), R), 1 / math.sqrt(D), window)
    return (q if dtype == torch.float32 else q.astype(np.float64)), Y


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [[4, 3, 9], [1, 70, 333]])
def test_few_rows(essa, ctx, dtype, rows):
    lens = [1, 50, 333]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=dtype, seed=50)
    _, none = _call(essa, ctx, c, rows, 6, dtype, 0)
    for window in (2 ** 31 - 1, 2 ** 31 - 2, 2 ** 31 - 64, 2 ** 30, 500):
        q, Y = _call(essa, ctx, c, rows, 6, dtype, window)
        check_attention(host(Y), q, c, [0, 1, 2], rows, 0.125, out_dtype=torch.float32)
        assert torch.equal(Y, none)


def test_much_work(essa, ctx):
    lens, rows = [3, 90, 3000], [200, 120, 3000]
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=torch.bfloat16, seed=52)
    _, none = _call(essa, ctx, c, rows, 6, torch.bfloat16, 0)
    assert (none[:197] == 0).all() and (none[197:200] != 0).any() and (none[200:230] == 0).all()
    for window in (2 ** 31 - 1, 2 ** 31 - 300, 3100):
        _, Y = _call(essa, ctx, c, rows, 6, torch.bfloat16, window)
        assert torch.equal(Y, none)


def test_wide_tables(essa, ctx):
    """A window below what the table could hold and above all that the pages do."""
    kv = essa.KvCache(ctx, 1, 1, 64, 2, page_tokens=32, max_seqs=1, max_tokens=2 ** 31 - 32)
    X = torch.randn(40, 1, 64, device="cuda")
    essa.essa_kv_extend(ctx, kv, i32([0]), i32([40]))
    batch = essa.KvBatch(i32([0]), starts([60]), 60)
    essa.essa_kv_append(ctx, kv, 0, X, X, essa.KvBatch(i32([0]), starts([40]), 40))
    Q = torch.randn(60, 1, 64, device="cuda")
    Y = [torch.full((60, 1, 64), 5.0, device="cuda") for _ in range(2)]
    essa.essa_kv_attention(ctx, kv, 0, Q, Y[0], batch, 0.125, window=2 ** 31 - 33)
    essa.essa_kv_attention(ctx, kv, 0, Q, Y[1], batch, 0.125)
    assert torch.equal(Y[0], Y[1]) and (Y[0][:20] == 0).all() and (Y[0][20:] != 0).any()
    kv.close()
