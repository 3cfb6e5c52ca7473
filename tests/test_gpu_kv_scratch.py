"""Attention's scratch is what its workgroups can fill."""
import pytest
import torch

from kv_helpers import i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,per_cu", [(64, 4), (128, 3)])
def test_scratch_of_a_small_call(essa, D, per_cu):
    """Two parts of 64 columns a workgroup, 256 CUs, a quarter more to grow in; a few MB for what the driver rounds to."""
    ctx = essa.Context(0)
    kv = essa.KvCache(ctx, 1, 1, D, 4, page_tokens=32, max_seqs=1, max_tokens=64)
    Q, batch = torch.zeros(1, 1, D, device="cuda"), essa.KvBatch(i32([0]))
    Y = torch.empty_like(Q)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    essa.essa_kv_attention(ctx, kv, 0, Q, Y, batch, 1.0)
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] <= 1.25 * 2 * 256 * per_cu * 64 * (D + 4) * 4 + 8 * 2 ** 20
    kv.close()
    ctx.close()
