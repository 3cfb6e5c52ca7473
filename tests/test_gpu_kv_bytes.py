"""The bytes that appends leave do not depend on how the rows came: all at once, in pieces, one by one."""
import numpy as np
import pytest
import torch

from kv_helpers import i32, starts, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,n", [(128, 70), (64, 64), (64, 33)])
def test_the_same_bytes(essa, D, n, dtype):
    ctx = essa.Context(0)
    hkv, g = 2, np.random.default_rng(3)
    K, V = values((n, hkv, D), g, dtype, outliers=True)[1], values((n, hkv, D), g, dtype)[1]
    pools = []
    for steps in ([n], [1] * n, [5, 32, 1, n - 38] if n > 38 else [31, n - 31], [1, n - 1], [n - 1, 1]):
        for alone in (True, False):                            # single rows without row starts, and with
            kv = essa.KvCache(ctx, 1, hkv, D, n_pages=4, page_tokens=32, max_seqs=1, max_tokens=96)
            kv.pool.zero_()
            at = 0
            for k in steps:
                essa.essa_kv_extend(ctx, kv, i32([0]), i32([k]))
                essa.essa_kv_append(ctx, kv, 0, K[at:at + k], V[at:at + k], essa.KvBatch(i32([0]), None if k == 1 and alone else starts([k]), k))
                at += k
            pools.append(kv.pool.clone())
            kv.close()
    assert all(torch.equal(p, pools[0]) for p in pools[1:]) and pools[0].any()
    ctx.close()
