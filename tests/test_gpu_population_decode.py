"""The example's recorded step owns every byte that it writes."""
import importlib.util
import os

import pytest
import torch

from kv_helpers import i32

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("population_decode", os.path.join(ROOT, "examples", "population_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_a_recorded_step_allocates_nothing_and_leaves_others_memory_alone(essa):
    mod, layers, hidden, n, steps = _example(), 2, 512, 6, 8
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        model = mod.Model(ctx, layers, hidden, 256, 8, 128, 2)
        kv = essa.KvCache(ctx, layers, model.kv_heads, 128, 12, page_tokens=32, max_seqs=n, max_tokens=64)
        buf, seqs, one = model.buffers(n), i32(range(n)), i32([1] * n)
        groups = model.groups(buf, i32([0, 0, 0, 1, 1, 1]))
        batch = essa.KvBatch(seqs)
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        begin = torch.randn(n, hidden, generator=g, device="cuda").bfloat16()

        def step():
            essa.essa_kv_extend(ctx, kv, seqs, one)
            model.forward(kv, buf, groups, batch)

        buf["x"].copy_(begin)
        want = []
        for _ in range(steps):                                 # call by call
            step()
            want.append(buf["x"].clone())
        torch.cuda.synchronize()
        essa.essa_kv_free(ctx, kv, seqs)
        made = torch.cuda.memory_stats()["allocation.all.allocated"]
        ctx.graph_begin()
        step()
        graph = ctx.graph_end()
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == made
        buf["x"].copy_(begin)
        others = []
        for t in range(steps):
            # memory of every size that a step could have used, handed out between the replays
            others += [torch.full((k,), 0x5a, dtype=torch.uint8, device="cuda") for k in (n * hidden * 4, n * hidden * 2, n * hidden, n * 4, 512) for _ in range(3)]
            graph.launch()
            torch.cuda.synchronize()
            assert torch.equal(buf["x"], want[t]), t
            assert all(bool((x == 0x5a).all()) for x in others), t
        graph.close()
        kv.close()
        ctx.close()
