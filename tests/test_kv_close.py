"""The check of attention's outputs itself (CPU): the kernels' arithmetic passes, a mistake of any kind does not."""
import math

import numpy as np
import pytest

import oracle as orc
from kv_close import check_close, levels

SHAPES = [(128, 28, 4, 400), (128, 28, 4, 2000), (64, 7, 1, 20011), (64, 6, 6, 130), (128, 3, 1, 1100), (128, 4, 2, 333)]


def _bf16(x):
    return ((np.ascontiguousarray(x, np.float32).view(np.uint32) + 0x8000) & 0xffff0000).view(np.float32)


def _case(D, hq, hkv, L, seed=0):
    g = np.random.default_rng(seed)
    K, V = (_bf16(g.standard_normal((L, hkv, D))) for _ in range(2))
    K[..., 3::29] += 5.0
    return _bf16(1.5 * g.standard_normal((1, hq, D))), _bf16(K), V


def _attention(q, K, V, scale, arithmetic, weights=None, values=None):
    """One row, all tokens: in 64 bits, or as either kernel rounds; weights, values: what a mistake makes of them."""
    half = lambda x: x.astype(np.float16).astype(np.float64)
    k, (codes, s, m) = levels(K)[0], orc.kv_quantise(V)
    s, m = (np.repeat(x.astype(np.float64), 64, -1) for x in (s, m))
    if values is not None:
        codes, s, m = (values(x) for x in (codes, s, m))
    y, g = np.zeros(q.shape), q.shape[1] // K.shape[1]
    for h in range(q.shape[1]):
        kk = half(k[:, h // g]) if arithmetic == "prompt" else k[:, h // g]
        z = scale * (kk @ q[0, h].astype(np.float64))
        p = np.exp(z - z.max())
        if weights is not None:
            p = weights(p)
        c, ss, mm = codes[:, h // g], s[:, h // g], m[:, h // g]
        if arithmetic == "stream":
            p = half(p * 2.0 ** 13)
            y[0, h] = ((half(p[:, None] * ss) * c).sum(0) + p @ mm) / p.sum()
        elif arithmetic == "prompt":
            p = half(p * 2.0 ** 4)
            y[0, h] = p @ half(mm + ss * c) / p.sum()
        else:
            y[0, h] = p @ (mm + ss * c) / p.sum()
    return y


@pytest.mark.parametrize("D,hq,hkv,L", SHAPES)
@pytest.mark.parametrize("arithmetic", ["exact", "stream", "prompt"])
def test_the_kernels_arithmetic_passes(D, hq, hkv, L, arithmetic):
    for seed in range(3):
        q, K, V = _case(D, hq, hkv, L, seed)
        scale = 1 / math.sqrt(D)
        share = check_close(_attention(q, K, V, scale, arithmetic), q, K, V, 1, scale)
        assert share < (1e-6 if arithmetic == "exact" else 0.6)


def _part(f, lo, n):
    """f on n tokens (or weights) from lo on."""
    def edit(x):
        x = x.copy()
        x[lo:lo + n] = f(x[lo:lo + n])
        return x
    return edit


@pytest.mark.parametrize("D,hq,hkv,L", SHAPES)
def test_mistakes_do_not(D, hq, hkv, L):
    q, K, V = _case(D, hq, hkv, L, 9)
    scale, at = 1 / math.sqrt(D), L // 2 // 64 * 64
    exact = _attention(q, K, V, scale, "exact")
    run = lambda **kw: _attention(q, K, V, kw.pop("scale", scale), "exact", **kw)
    wrong = {
        "zeros": 0 * exact, "1 % too large": 1.01 * exact, "0.02 added": exact + 0.02, "heads in another order": exact[:, ::-1], "channels turned by one": np.roll(exact, 1, 2),
        "a scale 2 % off": run(scale=1.02 * scale), "equal weights": run(weights=np.ones_like),
        "a block left out": run(weights=_part(np.zeros_like, at, 32)), "a stage left out": run(weights=_part(np.zeros_like, at, 64)),
        "the last token left out": run(weights=_part(np.zeros_like, L - 1, 1)) if L < 500 else None,
        "a block's values moved by a token": run(values=_part(lambda x: np.roll(x, 1, 0), at, 32)),
        "a part weighs 2 % more": run(weights=_part(lambda p: 1.02 * p, 0, L // 2)),
        "a block counted twice": run(weights=_part(lambda p: 2 * p, at, 32)),
    }
    for name, y in wrong.items():
        if y is None:
            continue
        print(name, flush=True)
        with pytest.raises(AssertionError):
            check_close(y, q, K, V, 1, scale)


def test_rows_windows_and_rows_that_see_nothing():
    g = np.random.default_rng(5)
    K, V, q = _bf16(g.standard_normal((30, 2, 64))), _bf16(g.standard_normal((30, 2, 64))), _bf16(g.standard_normal((40, 4, 64)))
    for window, causal in ((0, True), (7, True), (0, False)):
        y = orc.kv_attention(q.astype(np.float64), orc.kv_values(K), orc.kv_values(V), 40, 0.125, window, causal)[0]
        assert check_close(y, q, K, V, 40, 0.125, window, causal) < 1e-6
        for other in ((5, True), (0, True), (0, False)):
            if other != (window, causal):
                with pytest.raises(AssertionError):
                    check_close(y, q, K, V, 40, 0.125, *other)
        if causal:
            y[3, 1, 7] = 1e-9
            with pytest.raises(AssertionError):
                check_close(y, q, K, V, 40, 0.125, window, causal)
