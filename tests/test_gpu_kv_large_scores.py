"""Attention over the 4-bit cache where scores times scale are far past 2^22: single precision's steps of them are whole exponents there, but a row is still what its
largest score says.  Single tokens, several rows, prompts, fp32 queries, windows with sinks and trees."""
import math

import numpy as np
import pytest
import torch

import oracle as orc
from kv_close import levels, limits
from kv_helpers import Cache, host, i32, starts, values
from kv_masks import ancestors, random_tree, tree_words

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def check_largest(y, q, cache, seqs, rows, scale, masks, out_dtype, exact32):
    """Where a row's and head's largest score leads the next by more than the kernel's scores may be off by, and by 30 (weights below e^-30), the output is that token's
    value.  Scores: a key rounded to fp16 is off by 2^-11 of itself, two of them by 2^-10 sum |q k|, products of the codes that stand 128 too high add 2^-24 a step of 80 steps
    of 143 s |q|, which is less: 2^-9 sum |q k| together.  The value: a weight times a scale in fp16 2^-11 |s q|, or the value in fp16 2^-11 |v| (fp32 queries: a
    few 2^-24), what stands 1032 too high a few 2^-24 of 1032 s, the output's own rounding.  Returns the share of rows and heads that were looked at."""
    at, looked, of = 0, 0, 0
    for b, (s, n) in enumerate(zip(seqs, rows)):
        K, V = orc.kv_values(cache.K[0][s]), orc.kv_values(cache.V[0][s])
        codes, sc, mid = (x.astype(np.float64) for x in orc.kv_quantise(cache.V[0][s]))
        sc, mid = (np.repeat(x, orc.KV_GROUP, -1) for x in (sc, mid))
        g = q.shape[1] // K.shape[1]
        assert np.isfinite(y[at:at + n]).all(), ("not finite", s, np.argwhere(~np.isfinite(y[at:at + n]))[0])
        for h in range(q.shape[1]):
            k, qq = K[:, h // g], q[at:at + n, h].astype(np.float64)
            z, reach = scale * (qq @ k.T), abs(scale) * (np.abs(qq) @ np.abs(k).T)
            z = np.where(masks[b], z, -np.inf)
            for j in sorted({*range(0, n, max(1, n // 16)), n - 1}):
                if not masks[b][j].any():
                    assert (y[at + j, h] == 0).all()
                    continue
                of += 1
                best = int(z[j].argmax())
                if z[j, best] - np.delete(z[j], best).max(initial=-np.inf) <= 2.0 ** -9 * reach[j][masks[b][j]].max() + 30:
                    continue
                looked += 1
                v, size = V[best, h // g], np.abs(mid[best, h // g]) + np.abs(sc[best, h // g] * codes[best, h // g])
                bound = (2.0 ** -20 if exact32 else 2.0 ** -10) * size + 2.0 ** -12 * sc[best, h // g] * (2.0 ** -8 if exact32 else 1)
                if out_dtype == torch.bfloat16:
                    bound = bound + 2.0 ** -8 * (np.abs(v) + bound)
                err = np.abs(y[at + j, h] - v)
                assert (err <= bound).all(), ("row", j, "of entry", b, "head", h, "token", best, "error", err.max(), "bound", bound[err.argmax()])
        at += n
    return looked / of


SIZES = [(2e5, None), (3e7, None), (1e12, None), (1e20, None), (1e28, None), (5e32, None), (1.5, 1e9), (1.5, -1e20), (1e25, 1e-12)]      # of queries, scale


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q_scale,scale", SIZES)
@pytest.mark.parametrize("sort", ["single", "few rows", "prompts"])
@pytest.mark.parametrize("sight", ["causal", "window", "sinks", "tree"])
def test_large_scores(essa, ctx, dtype, q_scale, scale, sort, sight):
    g = np.random.default_rng(71)
    lens, rows, hq = {"single": ([900, 33, 1, 4000], None, 6), "few rows": ([300, 9, 2500], [20, 9, 3], 6), "prompts": ([420, 150, 700] * 3, [400, 90, 40] * 3, 12)}[sort]
    c = Cache(essa, ctx, lens, 2, 128 if sort != "few rows" else 64, 64, dtype=dtype, seed=72)
    D, per = c.kv.head_dim, [1] * len(lens) if rows is None else rows
    scale = 1 / math.sqrt(D) if scale is None else scale
    R = sum(per)
    q, qd = values((R, hq, D), g, dtype, scale=q_scale)
    window, sinks = {"window": (100, 0), "sinks": (60, 40), "tree": (0, 0), "causal": (0, 0)}[sight]
    trees = [ancestors(random_tree(g, n)) for n in per] if sight == "tree" else None
    tree = None if trees is None else tree_words(trees, 7)
    masks = [orc.kv_mask(L, n, window, sinks, None if trees is None else trees[i]) for i, (L, n) in enumerate(zip(lens, per))]
    batch = essa.KvBatch(i32(range(len(lens))), None if rows is None else starts(rows), R)
    print(dtype, q_scale, scale, sort, sight, flush=True)
    for out in (torch.float32, torch.bfloat16):
        Y = torch.full((R, hq, D), 5.0, device="cuda", dtype=out)
        essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, batch, scale, window, sinks=sinks, tree=tree)
        assert check_largest(host(Y), q, c, range(len(lens)), per, scale, masks, out, dtype == torch.float32) > 0.7
    c.kv.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [None, [70, 40]])
def test_rows_of_every_size_beside_each_other(essa, ctx, dtype, rows):
    """A row's result is its own, whatever the sizes of the rows beside it; a long sequence is many workgroups' parts."""
    lens, hq, D = [5000, 300], 4, 128
    c = Cache(essa, ctx, lens, 1, D, 64, dtype=dtype, seed=73)
    per = [1, 1] if rows is None else rows
    R = sum(per)
    q, qd = values((R, hq, D), np.random.default_rng(74), dtype)
    sizes = np.array([1e30, 1.5, 3e7, 1e15])
    q = q * sizes[(np.arange(R)[:, None] + np.arange(hq)) % 4][..., None]
    qd = torch.from_numpy(q.astype(np.float32)).cuda().to(dtype)
    q = host(qd)
    batch = essa.KvBatch(i32([0, 1]), None if rows is None else starts(rows), R)
    Y = torch.empty(R, hq, D, device="cuda")
    essa.essa_kv_attention(ctx, c.kv, 0, qd, Y, batch, 1 / math.sqrt(D))
    masks = [orc.kv_mask(L, n) for L, n in zip(lens, per)]
    y = host(Y)
    assert check_largest(y, q, c, [0, 1], per, 1 / math.sqrt(D), masks, torch.float32, dtype == torch.float32) > 0.5
    # Rows of ordinary size to their own limits.  (Not to the bits that they have alone: a column's maximum moves whenever one of its wave's does, and the
    # power of two that its weights are rounded at with it.)
    at, looked = 0, 0
    for s, n in enumerate(per):
        (k, _), (v, size) = levels(c.K[0][s]), levels(c.V[0][s])
        for j in range(n):
            for h in range(hq):
                if sizes[(at + j + h) % 4] != 1.5:
                    continue
                looked += 1
                qq = q[at + j, h].astype(np.float64)
                if dtype == torch.bfloat16:
                    want, limit = limits(qq, k[:, 0], v[:, 0], size[:, 0], masks[s][j], 1 / math.sqrt(D))
                    assert np.sqrt(np.square(y[at + j, h] - want).mean()) <= limit, (s, j, h)
                else:
                    want, mass, reach = (x[0, 0] for x in orc.kv_attention_masked(qq[None, None], k, v, masks[s][j:j + 1], 1 / math.sqrt(D)))
                    assert (np.abs(y[at + j, h] - want) <= (mass + np.abs(v).max()) * (2.0 ** -18 * (1 + reach) + lens[s] * 2.0 ** -24)).all(), (s, j, h)
        at += n
    assert looked == R * hq // 4
    c.kv.close()
