"""Row starts that do not ascend: every access stays inside, and what is not written is as it was."""
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


def _afterwards(essa, ctx, c, hq, dtype):
    """An ordinary call of the same cache is answered as ever."""
    n, D = len(c.lens), c.kv.head_dim
    rows = [min(3, x) for x in c.lens]
    q, qd = values((sum(rows), hq, D), np.random.default_rng(3), dtype)
    Y = torch.empty(sum(rows), hq, D, device="cuda")
    essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32(range(n)), starts(rows), sum(rows)), 0.1)
    check_attention(host(Y), q if dtype == torch.float32 else q.astype(np.float64), c, list(range(n)), rows, 0.1, out_dtype=torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("entries,R", [(8, 5), (40, 700), (300, 4000)])
def test_attention_of_more_rows_than_there_are(essa, ctx, dtype, entries, R):
    """0, R, 0, R, ..: every other entry names all rows.  The call does nothing."""
    hq, hkv, D = 6, 2, 64
    c = Cache(essa, ctx, [100 + i % 7 for i in range(entries)], hkv, D, 32, dtype=dtype, seed=1)
    Q = torch.randn(R, hq, D, device="cuda").to(dtype)
    Y = torch.full((R + 64, hq, D), 5.0, device="cuda", dtype=dtype)
    zigzag = i32([R * (i % 2) for i in range(entries + 1)])
    print("row starts", entries, R, dtype, flush=True)
    essa.essa_kv_attention(ctx, c.kv, 0, Q, Y[:R], essa.KvBatch(i32(range(entries)), zigzag, R), 0.1)
    torch.cuda.synchronize()
    assert (Y == 5).all()
    _afterwards(essa, ctx, c, hq, dtype)


@pytest.mark.parametrize("entries", [8, 40])
def test_append_and_read_of_rows_named_twice(essa, ctx, entries):
    """Every entry's tokens are some row's; nothing else of the pool changes, nothing past the rows is written."""
    hkv, D, R = 2, 64, 50
    c = Cache(essa, ctx, [100 + i % 7 for i in range(entries)], hkv, D, 32, dtype=torch.float32, seed=2)
    free = c.kv.refs == 0
    c.kv.pool[free] = 77
    zigzag = i32([R * (i % 2) for i in range(entries + 1)])
    batch = essa.KvBatch(i32(range(entries)), zigzag, R)
    X = torch.full((R + 8, hkv, D), 9.0, device="cuda")
    out = torch.full((2, R + 8, hkv, D), 5.0, device="cuda")
    essa.essa_kv_append(ctx, c.kv, 0, X[:R], X[:R], batch)
    essa.essa_kv_read(ctx, c.kv, 0, out[0, :R], out[1, :R], batch)
    torch.cuda.synchronize()
    assert (c.kv.pool[free] == 77).all() and (out[:, R:] == 5).all()
    for s in range(1, entries, 2):                             # entries that end before they begin have no rows
        n = c.lens[s]
        k, v = torch.empty(n, hkv, D, device="cuda"), torch.empty(n, hkv, D, device="cuda")
        essa.essa_kv_read(ctx, c.kv, 0, k, v, essa.KvBatch(i32([s]), starts([n]), n))
        assert not (k == 9).any() and not (v == 9).any()
