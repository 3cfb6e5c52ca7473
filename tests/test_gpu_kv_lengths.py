"""Lengths that no sequence can have, in a cache whose table is as wide as tables get: a sequence is never longer than all pages together."""
import pytest
import torch

from kv_helpers import i32, starts

pytestmark = pytest.mark.gpu


def test_spoiled_lengths_stay_inside(essa):
    """Positions are counted in 32 bits: with a table of 2^31 - 32 tokens, a length brought to no less than that let a block's first token wrap."""
    ctx = essa.Context(0)
    D, pages = 64, 4
    kv = essa.KvCache(ctx, 1, 1, D, pages, page_tokens=32, max_seqs=2, max_tokens=2 ** 31 - 32)
    kv.pool.zero_()
    for length in (2 ** 31 - 1, 2 ** 31 - 33, 32 * pages + 1):
        kv.table.fill_(-1)
        kv.refs.zero_()
        kv.len.fill_(length)
        for rows, batch in ((2, essa.KvBatch(i32([0, 1]))), (140, essa.KvBatch(i32([1, 0]), starts([133, 7]), 140))):
            print("length", length, "rows", rows, flush=True)
            X, Y = torch.zeros(rows, 1, D, device="cuda"), torch.full((rows, 1, D), 5.0, device="cuda")
            essa.essa_kv_append(ctx, kv, 0, X, X, batch)
            essa.essa_kv_read(ctx, kv, 0, Y, torch.empty_like(Y), batch)
            assert (Y == 0).all()
            for dtype in (torch.bfloat16, torch.float32):
                for window, causal in ((0, True), (40, True), (0, False)):
                    Y.fill_(5.0)
                    essa.essa_kv_attention(ctx, kv, 0, X.to(dtype), Y, batch, 1.0, window, causal)
                    assert (Y == 0).all()
        served = i32([0, 0])
        essa.essa_kv_extend(ctx, kv, i32([0, 1]), i32([0, 0]), served)
        assert served.tolist() == [0, 1] and kv.len.tolist() == [32 * pages] * 2
        kv.len.fill_(length)
        essa.essa_kv_fork(ctx, kv, i32([0]), i32([1]), served=served[:1])
        essa.essa_kv_compact(ctx, kv)
        essa.essa_kv_free(ctx, kv, i32([0, 1]))
        torch.cuda.synchronize()
        assert kv.len.tolist() == [0, 0] and (kv.table == -1).all()
    kv.close()
    ctx.close()
