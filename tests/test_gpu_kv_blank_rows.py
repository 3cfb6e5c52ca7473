"""Many rows that see nothing -- a prompt that found no pages, a sequence without tokens -- are zeros, and cost no more than if they saw something."""
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


@pytest.mark.parametrize("dtype,out", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("pad", [0, 1])
def test_zeros_beside_rows_that_see(essa, ctx, dtype, out, pad):
    lens, rows, hq = [200, 0, 33, 0, 500, 0], [4, 3000, 33, 65, 90, 64], 6
    c = Cache(essa, ctx, lens, 2, 64, 32, dtype=dtype, seed=81)
    seqs, R = [0, 1, 2, 3, 4, -2], sum(rows)
    q, qd = values((R, hq, 64), np.random.default_rng(82), dtype)
    flat = torch.full((R + 4, hq * 64 + pad), 5.0, device="cuda", dtype=out)
    Y = flat[2:R + 2, :hq * 64]
    essa.essa_kv_attention(ctx, c.kv, 0, qd.view(R, -1), Y, essa.KvBatch(i32(seqs), starts(rows), R), 0.125)
    y, at = host(Y.contiguous()).reshape(R, hq, 64), 0
    for s, n, length in zip(seqs, rows, lens):
        if s < 0 or length == 0:
            assert (y[at:at + n] == 0).all()
        else:
            check_close(y[at:at + n], q[at:at + n], c.K[0][s], c.V[0][s], n, 0.125, bf16_out=out == torch.bfloat16, which=[0, n // 2, n - 1])
        at += n
    assert (flat[:2] == 5).all() and (flat[R + 2:] == 5).all() and (flat[:, hq * 64:] == 5).all()


def test_many_entries_without_tokens(essa, ctx):
    """Entries on either side of what one workgroup does alone, past the first 64 of the list and among single rows."""
    n, hq = 300, 2
    rows = [1 if i % 7 else 60 + i % 11 for i in range(n)]
    kv = essa.KvCache(ctx, 1, 1, 64, 4, page_tokens=32, max_seqs=n, max_tokens=64)
    R = sum(rows)
    Q, Y = torch.randn(R, hq, 64, device="cuda").bfloat16(), torch.full((R, hq, 64), 5.0, device="cuda")
    essa.essa_kv_attention(ctx, kv, 0, Q, Y, essa.KvBatch(i32(range(n)), starts(rows), R), 0.125)
    assert (Y == 0).all()
    kv.close()


def test_skipped_prompts_cost_no_more_than_served_ones(essa, ctx):
    n, hq, hkv, D = 8000, 28, 4, 128
    kv = essa.KvCache(ctx, 1, hkv, D, 130, page_tokens=64, max_seqs=3, max_tokens=n)
    kv.pool.zero_()
    essa.essa_kv_extend(ctx, kv, i32([0]), i32([n]))
    Q = torch.randn(n, hq, D, device="cuda").bfloat16()
    Y = torch.empty_like(Q)
    times = []
    for seq in (0, -2, 1):
        batch = essa.KvBatch(i32([seq]), starts([n]), n)
        runs = []
        for _ in range(6):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            essa.essa_kv_attention(ctx, kv, 0, Q, Y, batch, 0.1)
            b.record()
            torch.cuda.synchronize()
            runs.append(a.elapsed_time(b))
        times.append(sorted(runs)[2])
    print("served, skipped, without tokens, ms:", times, flush=True)
    assert times[1] < times[0] and times[2] < times[0]
    kv.close()
