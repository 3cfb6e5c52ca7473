"""A decode step that was recorded before any prompt came does not keep prompts from coming: what it reserved is enough for them."""
import numpy as np
import pytest
import torch

from kv_close import check_close
from kv_helpers import Cache, host, i32, starts, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
def test_prompts_beside_a_recorded_step(essa, D):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        hq, hkv, lens = 14, 2, [4000, 300, 33]
        c = Cache(essa, ctx, lens, hkv, D, 64, dtype=torch.bfloat16, seed=71)
        g = np.random.default_rng(72)
        q1, q1d = values((1, hq, D), g, torch.bfloat16)
        qn, qnd = values((4300, hq, D), g, torch.bfloat16)
        y1, yn = torch.empty(1, hq, D, device="cuda"), torch.empty(4300, hq, D, device="cuda")
        one, many = essa.KvBatch(i32([2])), essa.KvBatch(i32([0, 1]), starts([4000, 300]), 4300)
        step = lambda: essa.essa_kv_attention(ctx, c.kv, 0, q1d, y1, one, 0.1)
        step()
        torch.cuda.synchronize()
        ctx.graph_begin()
        step()
        graph = ctx.graph_end()
        for _ in range(3):
            yn.fill_(5.0)
            essa.essa_kv_attention(ctx, c.kv, 0, qnd, yn, many, 0.1)
            y1.fill_(5.0)
            graph.launch()
            torch.cuda.synchronize()
            check_close(host(y1), q1, c.K[0][2], c.V[0][2], 1, 0.1)
            y = host(yn)
            check_close(y[:4000], qn[:4000], c.K[0][0], c.V[0][0], 4000, 0.1, which=[0, 1717, 3999])
            check_close(y[4000:], qn[4000:], c.K[0][1], c.V[0][1], 300, 0.1, which=[0, 299])
        graph.close()
        c.kv.close()
        ctx.close()
