"""The 4-bit key/value cache in plain numpy: the format, attention in 64 bits, and the bookkeeping of pages one step after
another.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

KV_GROUP, KV_BLOCK = 64, 32
KV_SKIPPED, KV_NO_PAGES, KV_TOO_LONG, KV_BAD_ENTRY = -1, -2, -3, -4


def kv_quantise(x):
    """x [..., D] -> (q [..., D] whole numbers, s [..., D / 64], m [..., D / 64]) with every operation in single precision."""
    x = np.asarray(x, np.float32)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // KV_GROUP, KV_GROUP))
    finite = np.isfinite(g).all(-1)
    g = np.clip(np.where(np.isfinite(g), g, np.float32(0)), np.float32(-32768), np.float32(32768))
    lo, hi = g.min(-1), g.max(-1)
    s = ((hi - lo) * (np.float32(1) / np.float32(15))).astype(np.float16).astype(np.float32)
    m = (lo + np.float32(8) * s).astype(np.float16).astype(np.float32)
    inverse = np.where(s > 0, np.float32(1) / np.where(s > 0, s, np.float32(1)), np.float32(0)).astype(np.float32)
    q = np.clip(np.rint((g - m[..., None]) * inverse[..., None]), -8, 7)
    s, m = np.where(finite, s, np.nan), np.where(finite, m, np.nan)
    return q.reshape(x.shape), s, m


def kv_values(x):
    """What the cache holds for x, in 64 bits."""
    q, s, m = kv_quantise(x)
    g = q.reshape(q.shape[:-1] + (q.shape[-1] // KV_GROUP, KV_GROUP)).astype(np.float64)
    return (m.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * g).reshape(q.shape)


def kv_attention(q, k, v, rows, scale, window=0, causal=True):
    """q [rows, Hq, D] (the last `rows` positions), k and v [L, Hkv, D] as the cache holds them, 64 bits.
    Returns (y [rows, Hq, D], mass [rows, Hq, D] = sum p |v|, reach [rows, Hq] = largest sum_c |scale q_c k_c| of a token seen)."""
    L, hkv, D = k.shape
    g = q.shape[1] // hkv
    y, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for j in range(rows):
        pos = L - rows + j
        lo, hi = 0, L
        if causal:
            hi = pos + 1
            if window > 0:
                lo = max(0, pos - window + 1)
        if lo >= hi:
            continue
        for h in range(q.shape[1]):
            kk, vv, qq = k[lo:hi, h // g], v[lo:hi, h // g], q[j, h].astype(np.float64)
            if not np.isfinite(qq).all():
                y[j, h] = np.nan
                continue
            z = scale * (kk @ qq)
            p = np.exp(z - z.max())
            p /= p.sum()
            y[j, h], mass[j, h] = p @ vv, p @ np.abs(vv)
            reach[j, h] = (np.abs(kk) @ np.abs(qq)).max() * abs(scale)
    return y, mass, reach


def kv_mask(L, rows, window=0, sinks=0, tree=None):
    """[rows, L] truth values: which tokens the last `rows` rows of a sequence of L tokens see.  tree: [rows, rows] truth values, row j sees row u."""
    base = L - rows
    seen = np.zeros((rows, L), bool)
    for j in range(rows):
        if tree is None:
            pos, end = base + j, base + j + 1
        else:
            mine = [u for u in range(rows) if tree[j][u] and base + u >= 0]
            pos, end = base + len([u for u in mine if u != j]), base
            seen[j, [base + u for u in mine]] = True
        for t in range(max(0, end)):
            if window == 0 or t > pos - window or t < sinks:
                seen[j, t] = True
    return seen


def kv_attention_masked(q, k, v, seen, scale):
    """As kv_attention, row j seeing the tokens seen[j]."""
    rows, hq, D = q.shape
    g = hq // k.shape[1]
    y, mass, reach = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for j in range(rows):
        at = np.flatnonzero(seen[j])
        if not len(at):
            continue
        for h in range(hq):
            one = kv_attention(q[j:j + 1, h:h + 1], k[at, h // g:h // g + 1], v[at, h // g:h // g + 1], 1, scale, causal=False)
            y[j, h], mass[j, h], reach[j, h] = one[0][0, 0], one[1][0, 0], one[2][0, 0]
    return y, mass, reach


class KvPages:
    """The bookkeeping, entry after entry.  `tokens[s]` is a list of anything (what the sequence's tokens are), so that contents can
    be followed through forks; pages are sets of indices only."""

    def __init__(self, n_pages, page_tokens, max_seqs, max_pages):
        self.page, self.max_pages, self.max_seqs = page_tokens, max_pages, max_seqs
        self.refs = [0] * n_pages
        self.pages = [[] for _ in range(max_seqs)]
        self.tokens = [[] for _ in range(max_seqs)]

    def _need(self, tokens):
        return -(-tokens // self.page)

    def _free(self):
        return [i for i, r in enumerate(self.refs) if r == 0]

    def extend(self, seqs, new):
        """new[i]: list of tokens, or a negative number."""
        free, served, asked, seen = self._free(), [], 0, set()
        for s, more in zip(seqs, new):
            n = more if isinstance(more, int) else len(more)
            if s < 0:
                served.append(KV_SKIPPED)
                continue
            if s >= self.max_seqs or s in seen or n < 0:
                seen.add(s)
                served.append(KV_BAD_ENTRY)
                continue
            seen.add(s)
            have = len(self.tokens[s])
            if self._need(have + n) > self.max_pages:
                served.append(KV_TOO_LONG)
                continue
            need = self._need(have + n) - self._need(have)
            at, asked = asked, asked + need
            if need and asked > len(free):
                served.append(KV_NO_PAGES)
                continue
            for p in free[at:asked]:
                self.pages[s].append(p)
                self.refs[p] = 1
            self.tokens[s] = self.tokens[s] + list(more)
            served.append(s)
        return served

    def fork(self, src, dst, lens=None):
        free, served, asked, seen, todo = self._free(), [], 0, set(), []
        refs = list(self.refs)
        sources = {a for a, b in zip(src, dst) if a >= 0 and a != b and 0 <= b < self.max_seqs and a < self.max_seqs}
        for i, (a, b) in enumerate(zip(src, dst)):
            if b < 0:
                served.append(KV_SKIPPED)
                continue
            if b >= self.max_seqs or a >= self.max_seqs or b in seen:
                seen.add(b)
                served.append(KV_BAD_ENTRY)
                continue
            seen.add(b)
            if a < 0:
                todo.append((b, [], [], None, self.pages[b]))
                served.append(b)
                continue
            have = len(self.tokens[a])
            n = have if lens is None or lens[i] < 0 else min(lens[i], have)
            full, copy = n // self.page, False
            if n % self.page:
                copy = a != b or (n < have and (refs[self.pages[a][full]] > 1 or a in sources))
            if copy:
                asked += 1
                if asked > len(free):
                    served.append(KV_NO_PAGES)
                    continue
            new = self.pages[a][:full]
            if n % self.page:
                new = new + [free[asked - 1] if copy else self.pages[a][full]]
            todo.append((b, new, self.tokens[a][:n], None, self.pages[b]))
            served.append(b)
        for b, new, _, _, old in todo:
            for p in new:
                self.refs[p] += 1
            for p in old:
                self.refs[p] -= 1
        for b, new, tokens, _, _ in todo:
            self.pages[b], self.tokens[b] = new, tokens
        return served

    def accept(self, seqs, rows, path, keep):
        """rows[b]: how many the entry has; path[b]: list of row numbers, of which the first keep[b] stay."""
        served, seen = [], set()
        for s, c, p, k in zip(seqs, rows, path, keep):
            if s < 0:
                served.append(KV_SKIPPED)
                continue
            bad = s >= self.max_seqs or s in seen
            seen.add(s)
            if not bad:
                base = len(self.tokens[s]) - c
                p = list(p[:max(k, 0)])
                bad = k < 0 or k > c or base < 0 or any(x < 0 or x >= c for x in p) or any(a >= b for a, b in zip(p, p[1:]))
                bad = bad or (c > 0 and any(self.refs[x] != 1 for x in self.pages[s][base // self.page:]))
            if bad:
                served.append(KV_BAD_ENTRY)
                continue
            self.tokens[s] = self.tokens[s][:base] + [self.tokens[s][base + x] for x in p]
            need = self._need(len(self.tokens[s]))
            for x in self.pages[s][need:]:
                self.refs[x] -= 1
            self.pages[s] = self.pages[s][:need]
            served.append(s)
        return served

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        high = [i for i, r in enumerate(self.refs) if r > 0 and i >= used]
        holes = [i for i, r in enumerate(self.refs) if r == 0 and i < used]
        where = {i: i for i, r in enumerate(self.refs) if r > 0}
        for a, b in zip(high, holes):
            where[a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.pages = [[where[p] for p in row] for row in self.pages]
        return used, [where.get(i, -1) for i in range(len(self.refs))]

    def table(self):
        t = np.full((self.max_seqs, self.max_pages), -1, np.int32)
        for s, row in enumerate(self.pages):
            t[s, :len(row)] = row
        return t
