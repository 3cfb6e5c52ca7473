"""Keys and values put into the 4-bit cache and read back, bit for bit against the format's definition."""
import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import Cache, host, i32, starts, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


def _f32(x):
    return x.astype(np.float32).astype(np.float64)


def _bf16(x):
    return host(torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16))


def _read(essa, ctx, kv, layer, seqs, rows, dtype=torch.float32):
    R = int(sum(rows))
    K = torch.full((R, kv.n_kv_heads, kv.head_dim), 7.0, device="cuda", dtype=dtype)
    V = torch.full_like(K, 7.0)
    essa.essa_kv_read(ctx, kv, layer, K, V, essa.KvBatch(i32(seqs), starts(rows), R))
    return host(K), host(V)


@pytest.mark.parametrize("D,hkv,page,dtype,lens", [
    (128, 4, 32, torch.bfloat16, [1, 31, 32, 33, 64, 100]),
    (64, 3, 64, torch.float32, [65, 2, 127, 128, 5]),
    (128, 1, 256, torch.float32, [300, 0, 17]),
    (64, 8, 128, torch.bfloat16, [1, 0, 1, 200]),
    (128, 2, 1024, torch.bfloat16, [1500, 700]),
])
def test_what_was_put_in_is_read_back(essa, ctx, D, hkv, page, dtype, lens):
    print("append / read D=%d heads=%d page=%d lens=%s" % (D, hkv, page, lens), flush=True)
    c = Cache(essa, ctx, lens, hkv, D, page, layers=2, dtype=dtype, seed=1)
    seqs = list(range(len(lens)))
    for layer in range(2):
        K, V = _read(essa, ctx, c.kv, layer, seqs, lens)
        Kb, Vb = _read(essa, ctx, c.kv, layer, seqs, lens, torch.bfloat16)
        at = 0
        for s, n in enumerate(lens):
            for got, got16, put in ((K, Kb, c.K), (V, Vb, c.V)):
                want = orc.kv_values(put[layer][s])
                np.testing.assert_array_equal(got[at:at + n], _f32(want))
                np.testing.assert_array_equal(got16[at:at + n], _bf16(want))
            at += n


def test_tokens_one_by_one_give_the_same_blocks(essa, ctx):
    """A token's codes lie among those of its neighbours: 70 single appends leave the bytes that one append of 70 rows leaves."""
    D, hkv, n = 128, 2, 70
    g = np.random.default_rng(3)
    K, Kd = values((n, hkv, D), g, torch.bfloat16, outliers=True)
    V, Vd = values((n, hkv, D), g, torch.bfloat16)
    pools = []
    for steps in ([1] * n, [n], [5, 32, 1, 32]):
        kv = essa.KvCache(ctx, 1, hkv, D, n_pages=4, page_tokens=32, max_seqs=1, max_tokens=96)
        kv.pool.zero_()
        at = 0
        for k in steps:
            essa.essa_kv_extend(ctx, kv, i32([0]), i32([k]))
            batch = essa.KvBatch(i32([0]), None if k == 1 else starts([k]), k)
            essa.essa_kv_append(ctx, kv, 0, Kd[at:at + k], Vd[at:at + k], batch)
            at += k
        k64, v64 = _read(essa, ctx, kv, 0, [0], [n])
        np.testing.assert_array_equal(k64, _f32(orc.kv_values(K)))
        np.testing.assert_array_equal(v64, _f32(orc.kv_values(V)))
        pools.append([_read(essa, ctx, kv, 0, [0], [n])])
        kv.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
def test_groups_at_the_edges_of_the_format(essa, ctx, dtype, D):
    """Constant groups, zeros, groups wider than fp16, subnormal ranges, infinities and NaN."""
    n, hkv = 40, 2
    g = np.random.default_rng(5)
    K, _ = values((n, hkv, D), g, dtype)
    K[0] = 0.0
    K[1] = 3.5
    K[2] *= 1e-7
    K[3] *= 1e30
    K[4] *= 20000.0
    K[5, 0, 7] = np.inf
    K[6, 1, D - 1] = -np.inf
    K[7, 0, 0] = np.nan
    K[8] = -40000.0
    K[9] = 1000.0 + K[9]
    K[10] *= 1e-38
    V, Vd = values((n, hkv, D), g, dtype)
    Kd = torch.from_numpy(K).cuda().to(dtype)
    K = host(Kd).astype(np.float32)
    kv = essa.KvCache(ctx, 1, hkv, D, n_pages=2, page_tokens=64, max_seqs=1, max_tokens=64)
    essa.essa_kv_extend(ctx, kv, i32([0]), i32([n]))
    essa.essa_kv_append(ctx, kv, 0, Kd, Vd, essa.KvBatch(i32([0]), starts([n]), n))
    k, v = _read(essa, ctx, kv, 0, [0], [n])
    np.testing.assert_array_equal(k, _f32(orc.kv_values(K)))
    np.testing.assert_array_equal(v, _f32(orc.kv_values(V)))
    assert np.isnan(k[5, 0, :64]).all() and np.isfinite(k[5, 1]).all() and np.isnan(k[7, 0, :64]).all()
    kv.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 0), (8, 1), (5, 3)])
def test_rows_at_any_distance(essa, ctx, dtype, pad, shift):
    """K and V as parts of wider rows (a fused projection's output), at offsets that no vector load is aligned to."""
    D, hkv, rows = 64, 3, [3, 0, 35]
    R, w = sum(rows), 3 * 64
    g = np.random.default_rng(6)
    x, _ = values((R, w + pad), g, dtype)
    y, _ = values((R, w + pad + 1), g, dtype)
    flat = torch.zeros(R * (w + pad) + shift, device="cuda", dtype=dtype)
    flat[shift:] = torch.from_numpy(x.reshape(-1)).cuda().to(dtype)
    Kd = flat[shift:].view(R, w + pad)[:, :w]
    Vd = torch.from_numpy(y).cuda().to(dtype)[:, 1:w + 1]
    kv = essa.KvCache(ctx, 1, hkv, D, n_pages=4, page_tokens=32, max_seqs=3, max_tokens=64)
    batch = essa.KvBatch(i32([2, 1, 0]), starts(rows), R)
    essa.essa_kv_extend(ctx, kv, i32([2, 1, 0]), i32(rows))
    essa.essa_kv_append(ctx, kv, 0, Kd, Vd, batch)
    out = torch.full((R, w + pad + 2), 9.0, device="cuda", dtype=dtype)
    out2 = torch.full((R, w + pad), 9.0, device="cuda", dtype=dtype)
    essa.essa_kv_read(ctx, kv, 0, out[:, 2 - (pad & 1):][:, :w], out2[:, :w], batch)
    rnd = _bf16 if dtype == torch.bfloat16 else _f32
    lo = 2 - (pad & 1)
    np.testing.assert_array_equal(host(out)[:, lo:lo + w], rnd(orc.kv_values(x[:, :w].reshape(R, hkv, D))).reshape(R, w))
    np.testing.assert_array_equal(host(out2)[:, :w], rnd(orc.kv_values(y[:, 1:w + 1].reshape(R, hkv, D))).reshape(R, w))
    assert (host(out)[:, :lo] == 9).all() and (host(out)[:, lo + w:] == 9).all() and (host(out2)[:, w:] == 9).all()
    kv.close()


def test_skipped_entries_and_rows_without_a_token(essa, ctx):
    lens = [40, 3, 70]
    c = Cache(essa, ctx, lens, 2, 64, 32, seed=8)
    before = c.kv.pool.clone()
    rows = [4, 50, 33, 2]
    seqs = [-1, 1, 5, 2]                                     # 5 is past max_seqs; sequence 1 has 3 tokens for 50 rows
    K, V = _read(essa, ctx, c.kv, 0, seqs, rows)
    assert (K[:4] == 0).all() and (V[:4] == 0).all() and (K[4:51] == 0).all() and (K[54:87] == 0).all()
    np.testing.assert_array_equal(K[51:54], _f32(orc.kv_values(c.K[0][1])))
    np.testing.assert_array_equal(V[87:], _f32(orc.kv_values(c.V[0][2][-2:])))
    X = torch.randn(sum(rows), 2, 64, device="cuda")
    essa.essa_kv_append(ctx, c.kv, 0, X, X, essa.KvBatch(i32([-1, -2, 5, -4]), starts(rows), sum(rows)))
    assert torch.equal(before, c.kv.pool)
    # rows in front of position 0 are left out, the three that are tokens go in
    essa.essa_kv_append(ctx, c.kv, 0, X, X, essa.KvBatch(i32([-1, 1, -1, -1]), starts(rows), sum(rows)))
    K, V = _read(essa, ctx, c.kv, 0, [1, 0, 2], lens[1:2] + lens[:1] + lens[2:])
    np.testing.assert_array_equal(K[:3], _f32(orc.kv_values(host(X)[51:54])))
    np.testing.assert_array_equal(V[3:43], _f32(orc.kv_values(c.V[0][0])))
    np.testing.assert_array_equal(K[43:], _f32(orc.kv_values(c.K[0][2])))


def test_pool_past_32_bits(essa, ctx):
    """A page's offset in bytes and a layer's within the page pass 2^32."""
    D, hkv, page, layers = 128, 8, 1024, 64
    kv = essa.KvCache(ctx, layers, hkv, D, n_pages=72, page_tokens=page, max_seqs=2, max_tokens=40 * page)
    size = kv.pool.numel()
    assert size > 2 ** 32 + 2 ** 30
    n = 70 * page // 2
    g = np.random.default_rng(9)
    K, Kd = values((3, hkv, D), g, torch.bfloat16)
    V, Vd = values((3, hkv, D), g, torch.bfloat16)
    essa.essa_kv_extend(ctx, kv, i32([0, 1]), i32([n, n]))
    essa.essa_kv_append(ctx, kv, layers - 1, Kd, Vd, essa.KvBatch(i32([1]), starts([3]), 3))
    k, v = _read(essa, ctx, kv, layers - 1, [1], [3])
    np.testing.assert_array_equal(k, _f32(orc.kv_values(K)))
    np.testing.assert_array_equal(v, _f32(orc.kv_values(V)))
    kv.close()


def test_refusals(essa, ctx):
    def refused(code, f):
        with pytest.raises(essa.EssaError) as ei:
            f()
        assert ei.value.code == code, ei.value
    refused(3, lambda: essa.KvCache(ctx, 1, 1, 96, 4))
    refused(2, lambda: essa.KvCache(ctx, 1, 1, 64, 4, page_tokens=48))
    refused(2, lambda: essa.KvCache(ctx, 0, 1, 64, 4))
    refused(2, lambda: essa.KvCache(ctx, 1, 1, 64, 4, max_seqs=5000))
    kv = essa.KvCache(ctx, 2, 2, 64, 4, page_tokens=32, max_seqs=3, max_tokens=64)
    X = torch.zeros(2, 2, 64, device="cuda")
    one = essa.KvBatch(i32([0, 1]))
    refused(2, lambda: essa.essa_kv_append(ctx, kv, 2, X, X, one))
    refused(2, lambda: essa.essa_kv_read(ctx, kv, -1, X, X, one))
    refused(2, lambda: essa.essa_kv_extend(ctx, kv, i32([0] * 4), i32([1] * 4)))
    refused(2, lambda: essa.essa_kv_attention(ctx, kv, 0, torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 3, 64, device="cuda"), one, 1.0))
    refused(1, lambda: essa.essa_kv_attention(ctx, kv, 0, X, X, one, 1.0, window=-1))
    refused(1, lambda: essa.essa_kv_attention(ctx, kv, 0, X, X, one, 1.0, window=3, causal=False))
    refused(1, lambda: essa.essa_kv_attention(ctx, kv, 0, X, X, one, float("nan")))
    other = essa.Context(0)
    refused(6, lambda: essa.essa_kv_append(other, kv, 0, X, X, one))
    other.close()
    with pytest.raises(TypeError):
        essa.essa_kv_append(ctx, kv, 0, X, X.bfloat16(), one)
    with pytest.raises(ValueError):
        essa.essa_kv_append(ctx, kv, 0, X[:1], X[:1], one)
    with pytest.raises(ValueError):
        essa.essa_kv_append(ctx, kv, 0, X.transpose(1, 2), X, one)
    with pytest.raises(ValueError):
        essa.KvBatch(i32([0, 1]), starts([1]), 1)
    kv.close()
