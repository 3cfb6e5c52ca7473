"""The largest scales: what the exponent of 2 cannot hold is refused, all below is computed with."""
import pytest
import torch

from kv_helpers import Cache, i32, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_scales_at_the_end_of_the_range(essa, dtype):
    ctx = essa.Context(0)
    c = Cache(essa, ctx, [40, 200], 2, 64, 32, dtype=dtype, seed=1)
    Q, rows = torch.zeros(90, 4, 64, device="cuda", dtype=dtype), [20, 70]
    batch = essa.KvBatch(i32([0, 1]), starts(rows), 90)
    Y = [torch.empty(90, 4, 64, device="cuda") for _ in range(2)]
    essa.essa_kv_attention(ctx, c.kv, 0, Q, Y[0], batch, 1.0)
    for scale in (2.3e38, -2.3e38, 1e-45):                    # queries of zero: every token weighs the same
        essa.essa_kv_attention(ctx, c.kv, 0, Q, Y[1].fill_(5.0), batch, scale)
        assert torch.equal(Y[0], Y[1]) and torch.isfinite(Y[1]).all(), scale
    for scale in (2.4e38, 3.4e38, -2.4e38, float("inf"), float("-inf"), float("nan")):
        Y[1].fill_(5.0)
        with pytest.raises(essa.EssaError) as ei:
            essa.essa_kv_attention(ctx, c.kv, 0, Q, Y[1], batch, scale)
        assert ei.value.code == 1 and (Y[1] == 5).all(), scale
    c.kv.close()
    ctx.close()
