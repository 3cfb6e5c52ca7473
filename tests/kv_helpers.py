"""Caches of random tokens for the GPU tests of the 4-bit key/value cache, and what their attention may be off by."""
import numpy as np
import torch

import essa_workloads as wl
import oracle as orc


def i32(a):
    return torch.tensor(list(a), dtype=torch.int32, device="cuda")


def starts(rows):
    return i32([0] + list(np.cumsum(rows)))


def host(t):
    if t.dtype == torch.bfloat16:
        return wl.bf16_bits_to_f32(t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)).astype(np.float64)
    return t.cpu().numpy().astype(np.float64) if t.dtype == torch.float32 else t.cpu().numpy()


def values(shape, g, dtype, scale=1.0, outliers=False):
    """Random values that are exactly of the type: (fp32 numpy, GPU tensor)."""
    x = (scale * g.standard_normal(shape)).astype(np.float32)
    if outliers:
        x[..., 3::29] += 5.0
    if dtype == torch.bfloat16:
        x = wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(x)).reshape(x.shape)
    return x, torch.from_numpy(x).cuda().to(dtype)


class Cache:
    """A cache whose sequence s holds lens[s] random tokens in every layer, put there in two turns; host copies of what was put in."""

    def __init__(self, essa, ctx, lens, hkv, D, page=32, layers=1, dtype=torch.float32, spare=3, seed=0, v_scale=1.0, edit=None):
        g = np.random.default_rng(seed)
        n = len(lens)
        self.lens = list(lens)
        self.kv = essa.KvCache(ctx, layers=layers, n_kv_heads=hkv, head_dim=D, n_pages=sum(-(-x // page) for x in lens) + spare, page_tokens=page, max_seqs=n + 2,
                               max_tokens=max(list(lens) + [1]) + 2 * page)
        self.K = [[None] * n for _ in range(layers)]
        self.V = [[None] * n for _ in range(layers)]
        for l in range(layers):
            for s in range(n):
                self.K[l][s] = values((lens[s], hkv, D), g, dtype, outliers=True)[0]
                self.V[l][s] = values((lens[s], hkv, D), g, dtype, scale=v_scale)[0]
                if edit:
                    edit(self.K[l][s], self.V[l][s], s)
                    if dtype == torch.bfloat16:
                        self.K[l][s], self.V[l][s] = (host(torch.from_numpy(x).to(dtype)).astype(np.float32) for x in (self.K[l][s], self.V[l][s]))
        seqs, done = i32(range(n)), [0] * n
        for turn in range(2):
            upto = [x // 3 if turn == 0 else x for x in lens]
            new = [u - d for u, d in zip(upto, done)]
            essa.essa_kv_extend(ctx, self.kv, seqs, i32(new))
            for l in range(layers):
                k = np.concatenate([self.K[l][s][done[s]:upto[s]] for s in range(n)])
                v = np.concatenate([self.V[l][s][done[s]:upto[s]] for s in range(n)])
                essa.essa_kv_append(ctx, self.kv, l, torch.from_numpy(k).cuda().to(dtype), torch.from_numpy(v).cuda().to(dtype),
                                    essa.KvBatch(seqs, starts(new), int(sum(new))))
            done = upto


def check_attention(got, q, cache, seqs, rows, scale, layer=0, window=0, causal=True, out_dtype=torch.bfloat16):
    """got and q [R, Hq, D] on the host, rows in the order of seqs; every element against the 64-bit value, within what the
    arithmetic can be off by:
      bf16 queries: weights, weights times scales, and the values of K and V held in 16 bits are off by 2^-11 of themselves each (a score
      then by 2^-11 of sum |q k|, a weight by e^(2 that)), weights below 2^-26 of the largest may be gone; fp32 sums are far below that.
      fp32 queries: a score is off by a few 2^-24 of sum |q k| a sum step, likewise everything else: 2^-18 covers D and the block sums,
      and a running sum of L terms L 2^-24.
    The output's own rounding (2^-9 for bf16) comes on top."""
    at = 0
    exact32 = q.dtype == np.float32
    for s, n in zip(seqs, rows):
        y = got[at:at + n]
        if s < 0:
            assert np.all(y == 0)
            at += n
            continue
        K, V = orc.kv_values(cache.K[layer][s]), orc.kv_values(cache.V[layer][s])
        want, mass, reach = orc.kv_attention(q[at:at + n], K, V, n, scale, window, causal)
        L = K.shape[0]
        # a weight's error meets s q and m apart: sum p |s q| <= sum p |v| + max |m|
        vmax = np.abs(np.where(np.isfinite(V), V, 0)).max() if L else 0.0
        amp = mass + vmax
        if exact32:
            bound = amp * (2.0 ** -18 * (1 + reach[..., None]) + L * 2.0 ** -24)
        else:
            bound = amp * (2.0 ** -9 + 2.0 ** -10 * reach[..., None]) + L * 2.0 ** -25 * vmax
        if out_dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.array_equal(np.isnan(y), np.isnan(want)), "NaN in other places"
        ok = np.isnan(want) | (np.abs(y - want) <= bound)
        assert ok.all(), (s, np.argwhere(~ok)[0], y[~ok][0], want[~ok][0], bound[~ok][0])
        # and the rms over a row's head, where not every error can be at its worst: half the bound's
        with np.errstate(invalid="ignore"):
            rms, lim = np.sqrt(np.nanmean((y - want) ** 2)) if y.size else 0.0, np.sqrt(np.nanmean(bound ** 2)) if y.size else 1.0
        assert not rms > lim / 2, (s, rms, lim)
        at += n
