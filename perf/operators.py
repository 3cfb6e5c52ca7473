"""The operators around the 4-bit key/value cache, as measurable cases.

Four kinds of case:

* "attend": attention of new rows over the cached tokens of their sequences (one layer), the tokens held in 4 bits.
* "append": new keys and values of one layer put into their sequences' pages in 4 bits, and the same rows read back as
  the values the cache now stands for.
* "fork": samples forked off prompts (whole pages shared, the partly filled last page copied in every layer), then
  lengthened by the tokens of a step, some of them freed again.
* "compact": the pages in use moved down into the holes below them, tables and counts renumbered.

With `own` false the passes are plain torch operations in 32 bits; with `own` true they are the framework's calls.

A group of 64 channels of one token and head is held as sixteen levels m + s (q - 8): with the values x clamped to
+-2^15, lo and hi their least and greatest, s = fp16((hi - lo) / 15), m = fp16(lo + 8 s) and
q = clamp(rint((x - m) (1 / s)) + 8, 0, 15), every operation in single precision; s = 0 gives q = 8.
"""
from __future__ import annotations

import math
import random

import torch

own = False

GROUP = 64          # channels that share a scale
BLOCK = 32          # tokens of a block, the unit that pages are made of


# ---------------------------------------------------------------------------------------------- cases
def _attend(name, hq, hkv, d, seqs, length, rows, x="bf16", page=64, layers=1, window=0, causal=True):
    return {"name": name, "kind": "attend", "hq": hq, "hkv": hkv, "d": d, "seqs": seqs, "len_lo": length[0], "len_hi": length[1], "rows_lo": rows[0],
            "rows_hi": rows[1], "x": x, "page": page, "layers": layers, "window": window, "causal": causal, "order": len(name)}


def _append(name, hkv, d, seqs, length, rows, x="bf16", page=64):
    return {"name": name, "kind": "append", "hq": hkv, "hkv": hkv, "d": d, "seqs": seqs, "len_lo": length[0], "len_hi": length[1], "rows_lo": rows[0],
            "rows_hi": rows[1], "x": x, "page": page, "layers": 1, "order": len(name)}


def _fork(name, layers, hkv, d, prompts, samples, length, new, page=64):
    return {"name": name, "kind": "fork", "layers": layers, "hkv": hkv, "d": d, "seqs": prompts, "samples": samples, "len_lo": length[0], "len_hi": length[1],
            "new": new, "page": page, "order": len(name)}


def _compact(name, layers, hkv, d, seqs, length, used, page=64):
    return {"name": name, "kind": "compact", "layers": layers, "hkv": hkv, "d": d, "seqs": seqs, "len_lo": length[0], "len_hi": length[1], "used": used,
            "page": page, "order": len(name)}


def listed():
    return [
        # one candidate answering one prompt, a token at a time: latency (28 query heads on 4 key heads, hidden 3584)
        _attend("decode_7b_1seq", 28, 4, 128, 1, (401, 401), (1, 1)),
        # the headline's decode step: 32 candidates x 8 samples, prompts and answers of every length
        _attend("decode_7b_256seqs", 28, 4, 128, 256, (130, 2100), (1, 1)),
        # long documents under the 72B-shaped model: few sequences, the work lies along the length, offsets past 32 bits
        _attend("decode_72b_long", 64, 8, 128, 4, (80000, 131072), (1, 1), layers=5),
        # a few drafted tokens of every sequence checked at once, local attention, pages of a single block
        _attend("verify_32b_window", 40, 8, 128, 48, (900, 9000), (2, 6), page=32, window=4096),
        # prompts entering the cache, whole or a piece behind what is there, beside sequences that decode: one batch
        _attend("mixed_7b_prompts", 28, 4, 128, 48, (64, 16000), (1, 2000)),
        # the tiny fp32 configuration: 8 heads of 64 with a key head each, several rows, odd lengths
        _attend("f32_tiny_heads", 8, 8, 64, 16, (3, 700), (1, 9), x="f32", page=32),
        # the decode step's new keys and values, one row a sequence
        _append("append_7b_256rows", 4, 128, 256, (130, 2100), (1, 1)),
        # a population's prompts: 64 sequences of about 512 rows, hidden 5120
        _append("append_32b_prompts", 8, 128, 64, (300, 800), (300, 724)),
        # eight samples of each of 32 candidates' prompts, 28 layers
        _fork("fork_7b_population", 28, 4, 128, 32, 8, (60, 900), 1),
        # one beam turning into four, a layer or two: latency of the bookkeeping
        _fork("fork_small", 2, 2, 64, 1, 4, (45, 45), 20, page=32),
        # a pool after many generations, two fifths of it holes, 28 layers
        _compact("compact_7b", 28, 4, 128, 96, (200, 2100), 0.6),
        # a small pool with a few holes
        _compact("compact_small", 2, 8, 64, 9, (1, 300), 0.8, page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend"] * 6 + ["append"] * 2 + ["fork", "compact"])
    d = rng.choice([64, 128, 128])
    page = rng.choice([32, 64, 64, 128, 256])
    hkv = rng.choice([1, 2, 3, 4, 5, 8])
    case = {"kind": kind, "d": d, "page": page, "hkv": hkv, "order": rng.randrange(1 << 20)}
    if kind == "attend":
        hq = hkv * rng.choice([1, 2, 3, 5, 7, 8, 16])
        sort = rng.choice(["decode", "decode", "few rows", "prompt"])
        x = rng.choice(["bf16", "bf16", "bf16", "f32"])
        hi = _log_int(rng, 20, 120000 if sort == "decode" else 12000)
        lo = rng.choice([1, _log_int(rng, max(1, hi // 30), hi)])
        seqs = _log_int(rng, 1, 300)
        rows = {"decode": (1, 1), "few rows": (1, rng.randint(2, 20)), "prompt": (rng.choice([1, lo]), rng.choice([hi, max(lo, hi // 5)]))}[sort]
        causal = rng.random() < 0.8
        case.update(hq=hq, seqs=seqs, len_lo=lo, len_hi=hi, rows_lo=rows[0], rows_hi=rows[1], x=x, layers=rng.randint(1, 3),
                    window=_log_int(rng, 1, 2 * hi) if causal and rng.random() < 0.25 else 0, causal=causal)
        while case["seqs"] > 1 and _too_much(case):
            case["seqs"] = case["seqs"] * 2 // 3
        while _too_much(case):
            case["len_hi"] = max(1, case["len_hi"] * 2 // 3)
            for bound in ("len_lo", "rows_lo", "rows_hi"):
                case[bound] = min(case[bound], case["len_hi"])
    elif kind == "append":
        rows = (1, 1) if rng.random() < 0.5 else (1, _log_int(rng, 2, 2000))
        seqs = _log_int(rng, 8, 400)
        case.update(hq=hkv, seqs=max(1, min(seqs, 15000 // rows[1])), len_lo=1, len_hi=max(rows[1], _log_int(rng, 30, 4000)), rows_lo=rows[0], rows_hi=rows[1],
                    x=rng.choice(["bf16", "bf16", "f32"]), layers=1)
    else:
        case.update(layers=_log_int(rng, 1, 28), seqs=_log_int(rng, 1, 64), len_lo=rng.choice([1, 30]), len_hi=_log_int(rng, 30, 1500))
        if kind == "fork":
            case.update(samples=rng.randint(1, 10), new=_log_int(rng, 1, 200))
        else:
            case.update(used=rng.uniform(0.3, 1.0))
        while _pool_bytes(case) > 2.5e9 and case["layers"] > 1:
            case["layers"] = case["layers"] * 2 // 3
        while _pool_bytes(case) > 2.5e9:
            case["seqs"] = max(1, case["seqs"] * 2 // 3)
    return case


def _lengths(case):
    """Cached tokens (the new ones among them) and new rows of every sequence: they belong to the case, not to the seed."""
    rng = random.Random(case["order"])
    lens, rows = [], []
    for i in range(case["seqs"]):
        length = _log_int(rng, case["len_lo"], case["len_hi"])
        new = 0
        if "rows_lo" in case:
            new = case["rows_lo"] if case["rows_lo"] == case["rows_hi"] or (i % 2 and case["rows_lo"] == 1) else rng.randint(case["rows_lo"], case["rows_hi"])
            new = min(new, length)
        lens.append(length)
        rows.append(new)
    return lens, rows


def _page_bytes(case):
    return case["layers"] * case["hkv"] * (case["page"] // BLOCK) * _block_bytes(case["d"])


def _block_bytes(d):
    return 2 * (BLOCK * d // 2 + BLOCK * (d // GROUP) * 4)      # codes, and two 16-bit numbers a group, of keys and of values


def _pages(case):
    return sum(-(-length // case["page"]) for length in _lengths(case)[0])


def _pool_bytes(case):
    if case["kind"] == "fork":
        per = 1 + -(-case["new"] // case["page"]) + 1
        return (_pages(case) + case["seqs"] * case["samples"] * per + 3) * _page_bytes(case)
    return int(_pages(case) / case["used"] + 2) * _page_bytes(case)


def _visible(case, length, new):
    """(row, token) pairs that attention looks at, and the tokens that any row looks at."""
    if not case["causal"]:
        return new * length, length
    pairs = 0
    for j in range(new):
        seen = length - new + j + 1
        pairs += min(seen, case["window"]) if case["window"] else seen
    first = max(0, length - new + 1 - case["window"]) if case["window"] else 0
    return pairs, (length - first) if new else 0


def _too_much(case):
    w = work(case)
    return w["flops"] > (2e11 if case["x"] == "f32" else 8e11) or w["bytes"] > 4e8 or case["seqs"] * case["hq"] * max(case["len_hi"] // 64, 1) > 400000


def work(case):
    kind, d = case["kind"], case["d"]
    lens, rows = _lengths(case)
    token = case["hkv"] * _block_bytes(d) / BLOCK
    size = 4 if case.get("x") == "f32" else 2
    if kind == "attend":
        pairs = toks = 0
        for length, new in zip(lens, rows):
            p, t = _visible(case, length, new)
            pairs, toks = pairs + p, toks + t
        return {"bytes": toks * token + 2 * sum(rows) * case["hq"] * d * size, "flops": 4 * d * case["hq"] * pairs}
    if kind == "append":
        return {"bytes": sum(rows) * (4 * case["hkv"] * d * size + 2 * token), "flops": 12 * sum(rows) * case["hkv"] * d}
    if kind == "fork":
        tail = sum(-(-(length % case["page"]) // BLOCK) for length in lens)
        table = 4 * (sum(lens) // case["page"] + 2 * case["seqs"]) * case["samples"]
        return {"bytes": 2 * case["samples"] * tail * case["layers"] * case["hkv"] * _block_bytes(d) + 2 * table, "flops": 0}
    used = _pages(case)
    total = int(used / case["used"] + 2)
    moved = used * (total - used) // total         # what lies above the last page in use, on average
    return {"bytes": 2 * moved * _page_bytes(case) + 8 * (used + total), "flops": 0}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _tokens(case, seed):
    """Keys and values of all tokens, sequence after sequence, and the new rows' queries.  Keys have channels that stand out, as a
    rotary or biased projection gives them; values have none; queries make the scores spread by a few units."""
    g = _gen(seed)
    lens, rows = _lengths(case)
    total, hkv, d = sum(lens), case["hkv"], case["d"]
    dtype = torch.float32 if case["x"] == "f32" else torch.bfloat16
    spread = torch.exp(0.4 * torch.randn(hkv, d, generator=g, device="cuda"))
    shift = 3.0 * torch.randn(hkv, d, generator=g, device="cuda") * (torch.rand(hkv, d, generator=g, device="cuda") < 0.06)
    K = torch.empty(total, hkv, d, device="cuda", dtype=dtype)
    V = torch.empty(total, hkv, d, device="cuda", dtype=dtype)
    for t in range(0, total, 65536):
        n = min(65536, total - t)
        K[t:t + n] = torch.randn(n, hkv, d, generator=g, device="cuda") * spread + shift
        V[t:t + n] = 0.7 * torch.randn(n, hkv, d, generator=g, device="cuda")
    Q = (1.4 * torch.randn(sum(rows), case["hq"], d, generator=g, device="cuda")).to(dtype)
    return K, V, Q


def _new_rows(case):
    """Indices of the new rows among all tokens (the last ones of each sequence)."""
    lens, rows = _lengths(case)
    out, at = [], 0
    for length, new in zip(lens, rows):
        out.append(torch.arange(at + length - new, at + length))
        at += length
    return torch.cat(out).cuda()


def _starts(rows):
    return torch.tensor([0] + torch.tensor(rows).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


def prepare(case, seed):
    if case["kind"] in ("attend", "append"):
        return _prepare_tokens(case, seed)
    return _prepare_pages(case, seed)


def _prepare_tokens(case, seed):
    lens, rows = _lengths(case)
    K, V, Q = _tokens(case, seed)
    state = {"case": case, "lens": lens, "rows": rows, "Q": Q}
    if case["kind"] == "append":
        pick = _new_rows(case)
        state["Knew"], state["Vnew"] = K[pick].contiguous(), V[pick].contiguous()
    if not own:
        if case["kind"] == "attend":
            state["K"], state["V"] = _pack_plain(K), _pack_plain(V)
        return state
    import paper_2507_04453_amd as essa
    ctx = essa.Context(0)
    n = len(lens)
    kv = essa.KvCache(ctx, layers=case["layers"], n_kv_heads=case["hkv"], head_dim=case["d"], n_pages=_pages(case) + 1, page_tokens=case["page"], max_seqs=n,
                      max_tokens=max(lens))
    seqs = torch.arange(n, dtype=torch.int32, device="cuda")
    layer = case["layers"] - 1
    # the history comes in two turns, so that the pages of different sequences lie among one another
    at = torch.tensor([0] + lens).cumsum(0)[:-1].tolist()
    done = [0] * n
    for turn in range(2):
        upto = [length // 2 if turn == 0 else length for length in lens]
        new = [u - s for u, s in zip(upto, done)]
        index = torch.cat([torch.arange(a + s, a + u) for a, s, u in zip(at, done, upto)]).cuda()
        essa.essa_kv_extend(ctx, kv, seqs, torch.tensor(new, dtype=torch.int32, device="cuda"))
        if len(index):
            essa.essa_kv_append(ctx, kv, layer, K[index], V[index], essa.KvBatch(seqs, _starts(new), len(index)))
        done = upto
    single = all(r == 1 for r in rows)
    state.update(ctx=ctx, kv=kv, layer=layer, essa=essa, scale=1.0 / math.sqrt(case["d"]),
                 batch=essa.KvBatch(seqs, None if single else _starts(rows), sum(rows)))
    if case["kind"] == "attend":
        state["Y"] = torch.empty_like(Q)
    else:
        state["Kback"], state["Vback"] = torch.empty_like(state["Knew"]), torch.empty_like(state["Vnew"])
    return state


def _pool_state(case, seed):
    """A pool of random pages, with the table, lengths and reference counts of its sequences.  What a page holds does not matter to the
    bookkeeping: a copy is that of its words, bit for bit, and they are compared as the whole numbers they are."""
    rng = random.Random(seed)
    lens, _ = _lengths(case)
    page, used = case["page"], _pages(case)
    if case["kind"] == "fork":
        n_pages, slots = _pool_bytes(case) // _page_bytes(case), case["seqs"] * (1 + case["samples"])
        max_tokens = max(lens) + case["new"]
    else:
        n_pages, slots, max_tokens = int(used / case["used"] + 2), case["seqs"], max(lens)
    max_pages = -(-max_tokens // page)
    order = rng.sample(range(n_pages), used)
    table = torch.full((slots, max_pages), -1, dtype=torch.int32)
    length = torch.zeros(slots, dtype=torch.int32)
    refs = torch.zeros(n_pages, dtype=torch.int32)
    at = 0
    for s, tokens in enumerate(lens):
        k = -(-tokens // page)
        table[s, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
        length[s] = tokens
        at += k
    refs[torch.tensor(order, dtype=torch.int64)] = 1
    return n_pages, slots, max_tokens, table.cuda(), length.cuda(), refs.cuda()


def _prepare_pages(case, seed):
    n_pages, slots, max_tokens, table, length, refs = _pool_state(case, seed)
    words = _block_bytes(case["d"]) // 4
    shape = (n_pages, case["layers"], case["hkv"], case["page"] // BLOCK, words)
    pool = torch.randint(-2 ** 31, 2 ** 31 - 1, shape, generator=_gen(seed), device="cuda", dtype=torch.int32)
    state = {"case": case, "pool": pool, "start": (table, length, refs), "max_pages": table.shape[1]}
    if case["kind"] == "fork":
        p, s = case["seqs"], case["samples"]
        dst = torch.arange(p, p * (1 + s), dtype=torch.int32)
        state["src"], state["dst"] = torch.arange(p, dtype=torch.int32).repeat_interleave(s).cuda(), dst.cuda()
        state["new"] = torch.full((p * s,), case["new"], dtype=torch.int32, device="cuda")
        state["gone"] = dst[::3].contiguous().cuda()
    if own:
        import paper_2507_04453_amd as essa
        ctx = essa.Context(0)
        kv = essa.KvCache(ctx, layers=case["layers"], n_kv_heads=case["hkv"], head_dim=case["d"], n_pages=n_pages, page_tokens=case["page"], max_seqs=slots,
                          max_tokens=max_tokens)
        kv.pool.view(torch.int32).copy_(pool.view(kv.pool.view(torch.int32).shape))
        state.update(ctx=ctx, kv=kv, essa=essa, pool=kv.pool.view(torch.int32).view(shape))
        if case["kind"] == "fork":
            state["served"] = [torch.empty_like(state["dst"]) for _ in range(2)]
        else:
            state["map"], state["used"] = torch.empty(n_pages, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    else:
        state["now"] = tuple(t.clone() for t in state["start"])
    return state


# ---------------------------------------------------------------------------------------------- passes
def run(state):
    return _RUN[state["case"]["kind"]](state)


def _run_attend(state):
    if own:
        case = state["case"]
        state["essa"].essa_kv_attention(state["ctx"], state["kv"], state["layer"], state["Q"], state["Y"], state["batch"], state["scale"], window=case["window"],
                                        causal=case["causal"])
        return state["Y"]
    return _attend_plain(state)


def _run_append(state):
    if own:
        essa = state["essa"]
        essa.essa_kv_append(state["ctx"], state["kv"], state["layer"], state["Knew"], state["Vnew"], state["batch"])
        essa.essa_kv_read(state["ctx"], state["kv"], state["layer"], state["Kback"], state["Vback"], state["batch"])
        return state["Kback"], state["Vback"]
    return tuple(_unpack_plain(_pack_plain(x)).to(x.dtype) for x in (state["Knew"], state["Vnew"]))


def _run_fork(state):
    # the samples of every generation start from the same prompts
    if own:
        essa, ctx, kv = state["essa"], state["ctx"], state["kv"]
        for now, start in zip((kv.table, kv.len, kv.refs), state["start"]):
            now.copy_(start)
        forked, longer = state["served"]
        essa.essa_kv_fork(ctx, kv, state["src"], state["dst"], served=forked)
        essa.essa_kv_extend(ctx, kv, state["dst"], state["new"], served=longer)
        essa.essa_kv_free(ctx, kv, state["gone"])
        return forked, longer, kv.table, kv.len, kv.refs, state["pool"]
    return _fork_plain(state)


def _run_compact(state):
    # a pool with the same holes every time
    if own:
        essa, ctx, kv = state["essa"], state["ctx"], state["kv"]
        for now, start in zip((kv.table, kv.len, kv.refs), state["start"]):
            now.copy_(start)
        essa.essa_kv_compact(ctx, kv, map_out=state["map"], used_out=state["used"])
        return state["used"], state["map"], kv.table, kv.len, kv.refs, state["pool"]
    return _compact_plain(state)


_RUN = {"attend": _run_attend, "append": _run_append, "fork": _run_fork, "compact": _run_compact}


# ---------------------------------------------------------------------------------------------- plain forms
def _pack_plain(x):
    """[tokens, heads, d] -> codes (8 bits each), scales and middles."""
    codes, scales, middles = [], [], []
    for part in x.split(65536):
        g = part.float().clamp(-32768.0, 32768.0).unflatten(2, (-1, GROUP))
        lo, hi = g.amin(3, keepdim=True), g.amax(3, keepdim=True)
        s = ((hi - lo) / 15.0).half().float()
        m = (lo + 8.0 * s).half().float()
        inverse = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
        codes.append((torch.round((g - m) * inverse) + 8.0).clamp(0.0, 15.0).to(torch.uint8).flatten(2))
        scales.append(s.squeeze(3).half())
        middles.append(m.squeeze(3).half())
    return torch.cat(codes), torch.cat(scales), torch.cat(middles)


def _unpack_plain(packed):
    codes, s, m = packed
    g = codes.unflatten(2, (-1, GROUP)).float() - 8.0
    return (m.float().unsqueeze(3) + s.float().unsqueeze(3) * g).flatten(2)


def _attend_plain(state):
    case, Q = state["case"], state["Q"]
    ratio, d = case["hq"] // case["hkv"], case["d"]
    scale = 1.0 / math.sqrt(d)
    out = torch.empty(Q.shape, device="cuda", dtype=torch.float32)
    at = row = 0
    for length, new in zip(state["lens"], state["rows"]):
        first = max(0, length - new + 1 - case["window"]) if case["window"] else 0
        k, v = (_unpack_plain(tuple(t[at + first:at + length] for t in state[name])) for name in ("K", "V"))
        q = Q[row:row + new].float()
        step = max(1, int(2e8) // max(1, new * ratio * (length - first)))          # key heads at a time: the scores are held whole
        mask = None
        if case["causal"] and (new > 1 or case["window"]):
            mine = torch.arange(length - new, length, device="cuda")[:, None]
            t = torch.arange(first, length, device="cuda")[None, :]
            mask = t > mine
            if case["window"]:
                mask = mask | (t <= mine - case["window"])
        for h in range(0, case["hkv"], step):
            heads = min(step, case["hkv"] - h)
            qh = q[:, h * ratio:(h + heads) * ratio].reshape(new, heads, ratio, d).permute(1, 2, 0, 3).reshape(heads, ratio * new, d)
            scores = torch.matmul(qh, k[:, h:h + heads].permute(1, 2, 0).contiguous()) * scale
            if mask is not None:
                scores = scores.view(heads, ratio, new, -1).masked_fill_(mask, float("-inf")).view(heads, ratio * new, -1)
            scores = torch.exp(scores - scores.amax(2, keepdim=True))
            o = torch.matmul(scores, v[:, h:h + heads].permute(1, 0, 2).contiguous()) / scores.sum(2, keepdim=True)
            out[row:row + new, h * ratio:(h + heads) * ratio] = o.view(heads, ratio, new, d).permute(2, 0, 1, 3).reshape(new, heads * ratio, d)
        at += length
        row += new
    return out.to(Q.dtype)


def _take_pages(refs, need):
    """The lowest free pages, one run for each entry of `need` in its order: (first of the run in the list, list)."""
    free = torch.nonzero(refs == 0).flatten()
    return torch.cumsum(need, 0) - need, free


def _fork_plain(state):
    case, pool = state["case"], state["pool"]
    table, length, refs = state["now"]
    for now, start in zip(state["now"], state["start"]):
        now.copy_(start)
    page = case["page"]
    src, dst, gone = state["src"].long(), state["dst"].long(), state["gone"].long()
    column = torch.arange(table.shape[1], device="cuda")
    # fork: full pages are shared, a partly filled one is copied as far as it is filled
    tokens = length[src].long()
    cut = tokens % page
    need = (cut > 0).long()
    first, free = _take_pages(refs, need)
    rows = table[src]
    full = column[None, :] < (tokens // page)[:, None]
    refs.index_add_(0, rows[full].long(), torch.ones_like(rows[full]))
    copied = torch.nonzero(need).flatten()
    new_pages, old_pages = free[first[copied]], rows[copied, tokens[copied] // page].long()
    for blocks in range(1, page // BLOCK + 1):
        these = torch.nonzero(-(-cut[copied] // BLOCK) == blocks).flatten()
        if len(these):
            pool[new_pages[these], :, :, :blocks] = pool[old_pages[these], :, :, :blocks]
    rows = torch.where(full, rows, torch.full_like(rows, -1))
    rows[copied, tokens[copied] // page] = new_pages.int()
    refs[new_pages] = 1
    table[dst], length[dst] = rows, tokens.int()
    forked = dst.int()
    # extend
    longer = tokens + state["new"].long()
    before, after = -(-tokens // page), -(-longer // page)
    first, free = _take_pages(refs, after - before)
    fresh = (column[None, :] >= before[:, None]) & (column[None, :] < after[:, None])
    which = free[(first[:, None] + column[None, :] - before[:, None])[fresh]]
    rows[fresh] = which.int()
    refs[which] = 1
    table[dst], length[dst] = rows, longer.int()
    # free
    held = table[gone]
    inside = column[None, :] < (-(-length[gone].long() // page))[:, None]
    refs.index_add_(0, held[inside].long(), -torch.ones_like(held[inside]))
    table[gone], length[gone] = -1, 0
    return forked, dst.int(), table, length, refs, pool


def _compact_plain(state):
    pool = state["pool"]
    table, length, refs = state["now"]
    for now, start in zip(state["now"], state["start"]):
        now.copy_(start)
    live = refs > 0
    index = torch.arange(len(refs), device="cuda")
    used = live.sum()
    high, holes = torch.nonzero(live & (index >= used)).flatten(), torch.nonzero(~live & (index < used)).flatten()
    for a, b in zip(high.split(64), holes.split(64)):
        pool[b] = pool[a]
    where = torch.where(live, index, torch.full_like(index, -1))
    where[high] = holes
    refs[holes] = refs[high]
    refs[high] = 0
    table.copy_(torch.where(table >= 0, where[table.clamp(min=0).long()].int(), table))
    return used.int().view(1), where.int(), table, length, refs, pool


# ---------------------------------------------------------------------------------------------- 64 bits
def _single(x):
    """What one operation in single precision gives: the result in 64 bits, rounded once."""
    return x.float().double()


def _levels_exact(x):
    """The values that a row of one head stands for in the cache, in 64 bits; x: [tokens, d]."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    for c in range(0, x.shape[1], GROUP):
        v = torch.clip(x[:, c:c + GROUP].double(), -32768.0, 32768.0)
        low = torch.min(v, 1, keepdim=True).values
        high = torch.max(v, 1, keepdim=True).values
        s = _single(_single(high - low) / 15).half().double()
        m = _single(low + 8 * s).half().double()
        q = torch.round(_single(_single(v - m) * _single(1 / torch.where(s == 0, torch.ones_like(s), s))))
        q = torch.where(s == 0, torch.zeros_like(q), torch.clip(q, -8, 7))
        out[:, c:c + GROUP] = m + s * q
    return out


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None                                    # whole numbers alone
    lens, rows = _lengths(case)
    K, V, Q = _tokens(case, seed)
    if case["kind"] == "append":
        pick = _new_rows(case)
        return tuple(torch.stack([_levels_exact(x[pick, h]) for h in range(case["hkv"])], 1) for x in (K, V))
    if work(case)["flops"] > 6e12:
        return None
    d, ratio = case["d"], case["hq"] // case["hkv"]
    out = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    for h in range(case["hkv"]):
        at = row = 0
        for length, new in zip(lens, rows):
            k, v = _levels_exact(K[at:at + length, h]), _levels_exact(V[at:at + length, h])
            for j in range(0, new, 512):
                n = min(512, new - j)
                last = torch.arange(length - new + j, length - new + j + n, device="cuda").view(n, 1)
                t = torch.arange(length, device="cuda").view(1, length)
                seen = torch.ones(n, length, dtype=torch.bool, device="cuda")
                if case["causal"]:
                    seen = t <= last
                    if case["window"]:
                        seen = seen & (last - t < case["window"])
                for r in range(ratio):
                    z = torch.mm(Q[row + j:row + j + n, h * ratio + r].double(), k.t().contiguous()) / math.sqrt(d)
                    z = torch.where(seen, z, torch.full_like(z, -math.inf))
                    z = torch.softmax(z, 1)
                    out[row + j:row + j + n, h * ratio + r] = torch.mm(z, v)
            at += length
            row += new
    return out
