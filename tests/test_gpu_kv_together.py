"""The cache's calls together: the example's population (prompts, forks, recorded steps, freeing, compaction), long lists of
entries, pools past 32 bits, empty calls, what a recording refuses."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import Cache, check_attention, host, i32, starts, values

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def test_the_example_recorded_and_call_by_call(essa):
    spec = importlib.util.spec_from_file_location("population_decode", os.path.join(ROOT, "examples", "population_decode.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    size = dict(candidates=3, samples=3, layers=2, hidden=512, kv_width=256, rank=8, prompt=70, steps=20, quiet=True)
    # recording runs nothing by itself, so both runs make the same number of steps
    a, b = mod.run(record=True, **size), mod.run(record=False, **size)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[2] == b[2]
    assert sorted(set(a[1].tolist())) == [0, 90]


def test_as_many_entries_as_there_can_be(essa, ctx):
    """4096 sequences: the longest list of entries, with rows of their own and without."""
    g = np.random.default_rng(1)
    n = 4096
    lens = [int(x) for x in g.integers(1, 40, n - 2)]
    c = Cache(essa, ctx, lens, 1, 64, 32, dtype=torch.bfloat16, seed=1)
    lens += [0, 0]
    c.K[0] += [np.zeros((0, 1, 64), np.float32)] * 2
    c.V[0] += [np.zeros((0, 1, 64), np.float32)] * 2
    pick = [int(x) for x in g.permutation(n)[:60]]
    for rows in (None, [int(x) for x in g.integers(0, 3, n)]):
        per = [1] * n if rows is None else rows
        R = sum(per)
        q, qd = values((R, 2, 64), g, torch.bfloat16)
        Y = torch.full_like(qd, 5.0)
        essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, essa.KvBatch(i32(range(n)), None if rows is None else starts(rows), R), 0.125)
        y, at = host(Y), np.concatenate([[0], np.cumsum(per)])
        assert not (y == 5).any()
        for s in pick:
            check_attention(y[at[s]:at[s + 1]], q[at[s]:at[s + 1]].astype(np.float64), c, [s], [per[s]], 0.125)


@pytest.mark.parametrize("rows", [3, 80])
def test_attention_in_a_pool_past_32_bits(essa, ctx, rows):
    """Every row sees its own token alone, in pages and layers whose offsets pass 2^32 bytes: the output is the value itself."""
    D, hkv, page, layers = 128, 8, 1024, 64
    kv = essa.KvCache(ctx, layers, hkv, D, n_pages=72, page_tokens=page, max_seqs=2, max_tokens=40 * page)
    assert kv.pool.numel() > 2 ** 32 + 2 ** 30
    g = np.random.default_rng(2)
    K, Kd = values((rows, hkv, D), g, torch.bfloat16)
    V, Vd = values((rows, hkv, D), g, torch.bfloat16)
    batch = essa.KvBatch(i32([1]), starts([rows]), rows)
    essa.essa_kv_extend(ctx, kv, i32([0, 1]), i32([35 * page, 35 * page]))
    essa.essa_kv_append(ctx, kv, layers - 1, Kd, Vd, batch)
    Y = torch.empty(rows, hkv, D, device="cuda")
    essa.essa_kv_attention(ctx, kv, layers - 1, Kd, Y, batch, 0.1, window=1)
    want = orc.kv_values(V)
    # one weight of 1: what is left is fp16's rounding of a value and of its scale (2^-11 each, of at most the group's largest)
    assert np.abs(host(Y) - want).max() <= 2.0 ** -9 * np.abs(want).max()
    kv.close()


def test_empty_calls(essa, ctx):
    kv = essa.KvCache(ctx, 1, 1, 64, 4, page_tokens=32, max_seqs=3, max_tokens=64)
    none, zero = i32([]), torch.empty(0, 1, 64, device="cuda")
    for batch in (essa.KvBatch(none), essa.KvBatch(i32([0, 1]), starts([0, 0]), 0)):
        essa.essa_kv_append(ctx, kv, 0, zero, zero, batch)
        essa.essa_kv_read(ctx, kv, 0, zero, zero, batch)
        essa.essa_kv_attention(ctx, kv, 0, zero, torch.empty_like(zero), batch, 1.0)
    essa.essa_kv_extend(ctx, kv, none, none)
    essa.essa_kv_fork(ctx, kv, none, none)
    essa.essa_kv_free(ctx, kv, none)
    essa.essa_kv_extend(ctx, kv, i32([0, 2]), i32([0, 0]))
    essa.essa_kv_compact(ctx, kv)
    assert kv.len.tolist() == [0, 0, 0] and not kv.refs.any() and (kv.table == -1).all()
    kv.close()


def test_a_recording_does_not_allocate(essa):
    """Attention whose scratch would have to grow is refused while a step is being recorded, and so is a new cache."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        kv = essa.KvCache(ctx, 1, 1, 64, 4, page_tokens=32, max_seqs=3, max_tokens=64)
        Q = torch.zeros(2, 1, 64, device="cuda")
        Y, batch = torch.empty_like(Q), essa.KvBatch(i32([0, 1]))
        torch.cuda.synchronize()
        ctx.graph_begin()
        try:
            for call in (lambda: essa.essa_kv_attention(ctx, kv, 0, Q, Y, batch, 1.0), lambda: essa.essa_kv_create(ctx, 1, 1, 64, 4)):
                with pytest.raises(essa.EssaError) as ei:
                    call()
                assert ei.value.code == 6
            Y.zero_()
        finally:
            graph = ctx.graph_end()
        graph.close()
        essa.essa_kv_attention(ctx, kv, 0, Q, Y, batch, 1.0)
        torch.cuda.synchronize()
        assert (Y == 0).all()                      # sequences of no tokens
        kv.close()
        ctx.close()
