"""Trees and masks for the tests of attention over the 4-bit cache, and its outputs held to 64 bits under them."""
import numpy as np
import torch

import oracle as orc
from kv_close import levels, limits


def random_tree(g, rows, chain=0.3):
    """Parents (-1: none), children behind their parents."""
    return [j - 1 if g.random() < chain else int(g.integers(-1, j)) for j in range(rows)]


def ancestors(parents):
    """[rows, rows] truth values: itself and its ancestors."""
    seen = np.zeros((len(parents), len(parents)), bool)
    for j, p in enumerate(parents):
        if p >= 0:
            seen[j] = seen[p]
        seen[j, j] = True
    return seen


def tree_words(per_entry, words, fill=0):
    """[rows, words] int64 of all entries' [rows, rows] truth values; fill: what bits past an entry's rows are (0 or 1)."""
    out = []
    for seen in per_entry:
        bits = np.full((len(seen), 64 * words), fill, np.uint8)
        n = min(len(seen), 64 * words)
        bits[:, :n] = seen[:, :n]
        out.append(np.packbits(bits, axis=1, bitorder="little").view(np.uint64).view(np.int64).reshape(len(seen), words))
    return torch.from_numpy(np.concatenate(out)).cuda()


def cut(seen, words):
    """What rows see of a tree whose rows have so many words."""
    seen = seen.copy()
    seen[:, 64 * words:] = False
    return seen


def check_masked(got, q, cache, seqs, rows, scale, masks, layer=0, out_dtype=torch.bfloat16, exact32=False):
    """got and q [R, Hq, D]; masks: for every entry [rows, len] truth values (None: skipped).  Every element within what the arithmetic can be off by
    (the bound is kv_helpers.check_attention's), and for bf16 queries every row's and head's rms within kv_close's limits."""
    at = 0
    for s, n, seen in zip(seqs, rows, masks):
        y, qq = got[at:at + n], q[at:at + n]
        at += n
        if s < 0 or seen is None:
            assert np.all(y == 0)
            continue
        K, V = orc.kv_values(cache.K[layer][s]), orc.kv_values(cache.V[layer][s])
        L = K.shape[0]
        want, mass, reach = orc.kv_attention_masked(qq, K, V, seen, scale)
        vmax = np.abs(np.where(np.isfinite(V), V, 0)).max() if L else 0.0
        amp = mass + vmax
        if exact32:
            bound = amp * (2.0 ** -18 * (1 + reach[..., None]) + L * 2.0 ** -24)
        else:
            bound = amp * (2.0 ** -9 + 2.0 ** -10 * reach[..., None]) + L * 2.0 ** -25 * vmax
        if out_dtype == torch.bfloat16:
            bound = bound + 2.0 ** -8 * (np.abs(want) + bound)
        assert np.array_equal(np.isnan(y), np.isnan(want)), ("NaN in other places", s, np.argwhere(np.isnan(y) != np.isnan(want))[:3])
        ok = np.isnan(want) | (np.abs(y - want) <= bound)
        assert ok.all(), (s, np.argwhere(~ok)[0], y[~ok][0], want[~ok][0], bound[~ok][0])
        assert (y[~seen.any(1)] == 0).all()
        if not exact32 and np.isfinite(K).all() and np.isfinite(V).all():
            (k, _), (v, size), g = levels(cache.K[layer][s]), levels(cache.V[layer][s]), q.shape[1] // K.shape[1]
            for j in sorted({0, n // 3, n - 1} if n else ()):
                for h in range(q.shape[1]):
                    if seen[j].any() and np.isfinite(qq[j, h]).all():
                        ref, limit = limits(qq[j, h].astype(np.float64), k[:, h // g], v[:, h // g], size[:, h // g], seen[j], scale)
                        if out_dtype == torch.bfloat16:
                            limit = np.hypot(limit, 2.0 ** -9 * np.sqrt(np.square(ref).mean()))
                        err = np.sqrt(np.square(y[j, h] - ref).mean())
                        assert err <= limit, ("row", j, "head", h, "rms error", err, "limit", limit)
