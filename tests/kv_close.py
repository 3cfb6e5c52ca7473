"""How far attention over the 4-bit cache may be from 64 bits, row by row and head by head, as an rms over the head's channels.

The kernels for bf16 queries round to 11 bits, each rounding by u = 2^-11 of the number at most (0.4 u rms) and independently of the others:
a token's weight, the weight times a value's scale, in calls of much work keys and values instead of the latter.  With p the softmax in 64 bits,
v = m + s q the token's values and y the output, a token's part of the output's error is therefore
  of its weight         p (v - y) u                (y by the sum of weights, which are summed as rounded)
  of weight times scale p s q u,  of its value     p v u
  of its score          p (v - y) d,  d = u sqrt(sum_c (scale q_c k_c)^2)
and the errors of the tokens add as squares: the limit is three times
  u sqrt(mean over c of sum_t p_t^2 [(|m| + |s q| + |y|)^2 + ((|v| + |y|) sqrt(sum_c (scale q k)^2))^2])
where 0.4 to 0.6 times is expected.  p_t is taken as 2^-17 of the largest at least (weights are above 2^-28 of it or gone).  The output's own rounding comes on top.
"""
import numpy as np

import oracle as orc

U, TIMES = 2.0 ** -11, 3.0


def levels(x):
    """(values, |m| + |s q|) of rows [L, heads, D] as the cache holds them."""
    q, s, m = orc.kv_quantise(x)
    g = q.reshape(q.shape[:-1] + (q.shape[-1] // orc.KV_GROUP, orc.KV_GROUP)).astype(np.float64)
    m, s = m.astype(np.float64)[..., None], s.astype(np.float64)[..., None]
    return (m + s * g).reshape(q.shape), (np.abs(m) + np.abs(s * g)).reshape(q.shape)


def limits(q, k, v, size, seen, scale):
    """q [D], k, v, size [L, D] of one head, seen: slice of tokens -> (y, limit of the rms over D)."""
    kk, vv, aa = k[seen], v[seen], size[seen]
    z = scale * (kk @ q)
    p = np.exp(z - z.max())
    p /= p.sum()
    y = p @ vv
    w = np.maximum(p, p.max() * 2.0 ** -17) ** 2
    r = np.square(scale * kk * q).sum(1)
    part = w @ np.square(aa + np.abs(y)) + (w * r) @ np.square(np.abs(vv) + np.abs(y))
    return y, TIMES * U * np.sqrt(part.mean())


def check_close(got, q, K, V, rows, scale, window=0, causal=True, bf16_out=False, which=None):
    """got, q [rows, Hq, D]: the last rows of a sequence whose keys and values were K, V [L, Hkv, D]; which: only these rows.  Returns the largest
    share of its limit that an rms had."""
    (k, _), (v, size), L, worst = levels(K), levels(V), K.shape[0], 0.0
    g = q.shape[1] // K.shape[1]
    for j in range(rows) if which is None else which:
        pos = L - rows + j
        lo, hi = (max(0, pos - window + 1) if window else 0, pos + 1) if causal else (0, L)
        for h in range(q.shape[1]):
            if hi <= lo:
                assert (got[j, h] == 0).all(), ("row", j, "head", h, "sees nothing")
                continue
            y, limit = limits(q[j, h].astype(np.float64), k[:, h // g], v[:, h // g], size[:, h // g], slice(lo, hi), scale)
            if bf16_out:
                limit = np.hypot(limit, 2.0 ** -9 * np.sqrt(np.square(y).mean()))
            err = np.sqrt(np.square(got[j, h] - y).mean())
            assert err <= limit, ("row", j, "head", h, "rms error", err, "limit", limit, "rms of the output", np.sqrt(np.square(y).mean()))
            worst = max(worst, err / limit)
    return worst
