"""Scoring answers and drafting ahead over the 4-bit key/value cache, as measurable cases.

Four kinds of case:

* "logp": log probabilities of given tokens from a row of logits, the row's entropy, and its most probable tokens.
* "sinks": attention over the cache through a sliding window, with a few first tokens that stay visible.
* "tree": attention of a tree of drafted tokens over the cache: every row sees what was there before the tree, and its ancestors.
* "accept": the drafted rows of several layers put into the cache, the path that was right kept, the rest given back, and the kept
  rows read back.

With `own` false the passes are plain torch operations in 32 bits; with `own` true they are the framework's calls.

A group of 64 channels of one token and head is held as sixteen levels m + s q: with the values x clamped to +-2^15, lo and hi their least
and greatest, r = 1 / 15 in single precision, s = fp16((hi - lo) r), m = fp16(lo + 8 s) and q = clamp(rint((x - m) (1 / s)), -8, 7), every
operation in single precision; s = 0 gives q = 0.
"""
from __future__ import annotations

import math
import random

import torch

own = False

GROUP = 64          # channels that share a scale
BLOCK = 32          # tokens of a block, the unit that pages are made of


# ---------------------------------------------------------------------------------------------- cases
def _logp(name, rows, vocab, given, top, x="bf16", pad=0, scale=1.0, banned=0.0):
    return {"name": name, "kind": "logp", "rows": rows, "vocab": vocab, "given": given, "top": top, "x": x, "pad": pad, "scale": scale, "banned": banned}


def _attend(name, kind, hq, hkv, d, seqs, length, rows, x="bf16", page=64, window=0, sinks=0):
    return {"name": name, "kind": kind, "hq": hq, "hkv": hkv, "d": d, "seqs": seqs, "len_lo": length[0], "len_hi": length[1], "rows_lo": rows[0],
            "rows_hi": rows[1], "x": x, "page": page, "layers": 1, "window": window, "sinks": sinks, "order": len(name)}


def _accept(name, layers, hkv, d, seqs, length, rows, x="bf16", page=64):
    return {"name": name, "kind": "accept", "hq": hkv, "hkv": hkv, "d": d, "seqs": seqs, "len_lo": length[0], "len_hi": length[1], "rows_lo": rows[0],
            "rows_hi": rows[1], "x": x, "page": page, "layers": layers, "window": 0, "sinks": 0, "order": len(name)}


def listed():
    return [
        # one answer, the token it has just been given: latency
        _logp("logp_1row", 1, 152064, 1, 5),
        # the headline's decode step, 32 candidates x 8 samples, with the alternatives that a log of answers keeps
        _logp("logp_256rows", 256, 152064, 1, 20),
        # prompts and answers of a population scored after the fact: nothing but the tokens that are there
        _logp("logp_score_8192rows", 8192, 152064, 1, 0),
        # four choices a question, some tokens forbidden, a temperature, fp32 logits in rows of an odd length
        _logp("logp_f32_choices", 301, 32001, 4, 8, x="f32", pad=3, scale=1.0 / 0.7, banned=0.3),
        # the headline's decode step with answers of any length and a bounded window
        _attend("sinks_7b_256seqs", "sinks", 28, 4, 128, 256, (200, 16000), (1, 1), window=1024, sinks=4),
        # one very long document under the 72B-shaped model: little is seen of it
        _attend("sinks_72b_1seq", "sinks", 64, 8, 128, 1, (100001, 100001), (1, 1), page=128, window=4096, sinks=64),
        # prompts of every length entering the cache through the window
        _attend("sinks_32b_prompts", "sinks", 40, 8, 128, 12, (90, 6000), (90, 6000), window=1000, sinks=16),
        # a tree of 26 drafted tokens for each of 48 answers
        _attend("tree_7b_48seqs", "tree", 28, 4, 128, 48, (130, 4000), (26, 26)),
        # one answer, a large tree: latency
        _attend("tree_72b_1seq", "tree", 64, 8, 128, 1, (2049, 2049), (63, 63)),
        # the tiny fp32 configuration, trees of more than one word of ancestors
        _attend("tree_f32_heads", "tree", 8, 8, 64, 16, (140, 900), (5, 130), x="f32", page=32),
        # trees of 64 answers in four layers
        _accept("accept_7b_64seqs", 4, 4, 128, 64, (70, 3000), (8, 63)),
        # one small tree: latency of the calls
        _accept("accept_1seq", 2, 2, 64, 1, (45, 45), (9, 9), page=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["logp"] * 3 + ["sinks"] * 3 + ["tree"] * 3 + ["accept"])
    if kind == "logp":
        vocab = rng.choice([_log_int(rng, 100, 300000), _log_int(rng, 30000, 260000)])
        x = rng.choice(["bf16", "bf16", "f32"])
        rows = _log_int(rng, 1, max(1, min(16000, int((1.2e9 if x == "bf16" else 6e8) / vocab))))
        top = min(rng.choice([0, rng.randint(1, 8), rng.randint(1, 64)]), vocab // 8)
        if top:
            rows = min(rows, max(1, int(1e8 / vocab)))
        return {"kind": kind, "rows": rows, "vocab": vocab, "given": rng.choice([1, 1, rng.randint(2, 16)]), "top": top, "x": x,
                "pad": rng.choice([0, 0, rng.randint(1, 40)]), "scale": rng.choice([1.0, rng.uniform(0.3, 2.0)]), "banned": rng.choice([0.0, 0.0, rng.uniform(0.1, 0.6)])}
    d, hkv = rng.choice([64, 128, 128]), rng.choice([1, 2, 3, 4, 5, 8])
    case = {"kind": kind, "d": d, "hkv": hkv, "hq": hkv * rng.choice([1, 2, 3, 5, 7, 8, 16]), "page": rng.choice([32, 64, 64, 128, 256]), "layers": 1, "window": 0, "sinks": 0,
            "x": rng.choice(["bf16", "bf16", "bf16", "f32"]), "order": rng.randrange(1 << 20)}
    if kind == "sinks":
        sort = rng.choice(["decode", "decode", "few rows", "prompt"])
        hi = _log_int(rng, 40, 60000 if sort == "decode" else 6000)
        lo = rng.choice([1, _log_int(rng, max(1, hi // 30), hi)])
        rows = {"decode": (1, 1), "few rows": (1, rng.randint(2, 20)), "prompt": (rng.choice([1, lo]), rng.choice([hi, max(lo, hi // 5)]))}[sort]
        case.update(seqs=_log_int(rng, 1, 300), len_lo=lo, len_hi=hi, rows_lo=rows[0], rows_hi=rows[1], window=_log_int(rng, 1, min(hi, 8000)), sinks=_log_int(rng, 1, 300))
    elif kind == "tree":
        rows = _log_int(rng, 2, 200)
        hi = _log_int(rng, rows, 8000)
        some = rng.random() < 0.25
        case.update(seqs=_log_int(rng, 1, 120), len_lo=rows, len_hi=max(rows, hi), rows_lo=rng.choice([1, rows]), rows_hi=rows,
                    window=_log_int(rng, 1, 4000) if some else 0, sinks=rng.choice([0, rng.randint(1, 100)]) if some else 0)
    else:
        rows = _log_int(rng, 2, 200)
        case.update(hq=hkv, seqs=_log_int(rng, 1, max(1, min(200, 4000 // rows))), len_lo=rows, len_hi=max(rows, _log_int(rng, 30, 4000)), rows_lo=rng.choice([1, rows]), rows_hi=rows,
                    layers=rng.randint(1, 4))
        return case
    while case["seqs"] > 1 and _too_much(case):
        case["seqs"] = case["seqs"] * 2 // 3
    while _too_much(case):
        case["len_hi"] = max(1, case["len_hi"] * 2 // 3)
        for bound in ("len_lo", "rows_lo", "rows_hi"):
            case[bound] = min(case[bound], case["len_hi"])
    return case


def _lengths(case):
    """Cached tokens (the new ones among them) and new rows of every sequence: they belong to the case, not to the seed."""
    rng = random.Random(case["order"])
    lens, rows = [], []
    for _ in range(case["seqs"]):
        length = _log_int(rng, case["len_lo"], case["len_hi"])
        lens.append(length)
        rows.append(min(length, rng.randint(case["rows_lo"], case["rows_hi"])))
    return lens, rows


def _trees(case):
    """Every row's parent among its sequence's rows (-1: the token before the tree), children behind their parents: trees as a drafting
    program lays them out once, broad at the root."""
    rng = random.Random(case["order"] + 1)
    return [[j - 1 if rng.random() < 0.3 else rng.randrange(-1, j) for j in range(n)] for n in _lengths(case)[1]]


def _paths(case):
    """The rows of each tree that turned out right: a path from its root, in order."""
    rng = random.Random(case["order"] + 2)
    out = []
    for parents in _trees(case):
        at, walk = rng.randrange(len(parents)), []
        while at >= 0:
            walk.append(at)
            at = parents[at]
        out.append(walk[::-1])
    return out


def _words(case):
    return -(-max(_lengths(case)[1]) // 64)


def _ancestors(parents):
    """Row after row, the set of rows that it sees (itself and its ancestors) as a number."""
    seen = []
    for j, p in enumerate(parents):
        seen.append((1 << j) | (seen[p] if p >= 0 else 0))
    return seen


def _token_bytes(case):
    return case["hkv"] * 2 * (case["d"] // 2 + case["d"] // GROUP * 4)         # codes, and two 16-bit numbers a group, of keys and of values


def _visible(case, length, new, seen):
    """(row, token) pairs that attention looks at, and the tokens that any row looks at."""
    base, pairs, first = length - new, 0, length
    for j in range(new):
        drafted = bin(seen[j]).count("1") if seen else j + 1
        at = base + drafted - 1
        lo = min(max(0, at - case["window"] + 1), base) if case["window"] else 0
        if not seen:
            lo = max(0, at - case["window"] + 1) if case["window"] else 0
            pairs += at + 1 - lo + min(lo, case["sinks"])
        else:
            pairs += base - lo + min(lo, case["sinks"]) + drafted
        first = min(first, lo)
    return pairs, length - first + min(first, case["sinks"])


def _too_much(case):
    w = work(case)
    return w["flops"] > (1e11 if case["x"] == "f32" else 6e11) or w["bytes"] > 1.5e8 or sum(r * n for n, r in zip(*_lengths(case))) * case["hq"] > 4e9


def work(case):
    size = 4 if case["x"] == "f32" else 2
    if case["kind"] == "logp":
        out = case["given"] * 8 + 4 + case["top"] * 8
        return {"bytes": case["rows"] * (case["vocab"] * size + out), "flops": 6 * case["rows"] * case["vocab"]}
    lens, rows = _lengths(case)
    d, token = case["d"], _token_bytes(case)
    if case["kind"] == "accept":
        kept = sum(len(p) for p in _paths(case))
        return {"bytes": case["layers"] * (2 * sum(rows) * case["hkv"] * d * size + sum(rows) * token + 2 * kept * token + kept * (token + 2 * case["hkv"] * d * size)),
                "flops": 12 * case["layers"] * sum(rows) * case["hkv"] * d}
    trees = [_ancestors(p) for p in _trees(case)] if case["kind"] == "tree" else [None] * len(lens)
    pairs = toks = 0
    for length, new, seen in zip(lens, rows, trees):
        p, t = _visible(case, length, new, seen)
        pairs, toks = pairs + p, toks + t
    words = 8 * sum(rows) * _words(case) if case["kind"] == "tree" else 0
    return {"bytes": toks * token + 2 * sum(rows) * case["hq"] * d * size + words, "flops": 4 * d * case["hq"] * pairs}


# ---------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dtype(case):
    return torch.float32 if case["x"] == "f32" else torch.bfloat16


def _logits(case, seed):
    """Logits as a head gives them: most tokens near one another, some that stand out, each row of a sharpness of its own; `banned` of the
    tokens are forbidden (-inf), the given ones never."""
    g = _gen(seed)
    rows, vocab = case["rows"], case["vocab"]
    wide = torch.empty(rows, vocab + case["pad"], device="cuda", dtype=_dtype(case))
    sharp = torch.rand(rows, 1, generator=g, device="cuda") * 3.0 + 0.7
    tokens = torch.randint(0, vocab, (rows, case["given"]), generator=g, device="cuda")
    step = max(1, int(2e8) // vocab)
    for i in range(0, rows, step):
        n = min(step, rows - i)
        x = torch.randn(n, vocab, generator=g, device="cuda").mul_(sharp[i:i + n])
        if case["banned"]:
            out = torch.rand(n, vocab, generator=g, device="cuda") < case["banned"]
            out.scatter_(1, tokens[i:i + n], False)
            x.masked_fill_(out, float("-inf"))
        wide[i:i + n, :vocab] = x
    top = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    some = torch.rand(rows, generator=g, device="cuda") < 0.7                  # the token that the row is about, and often the one that was given
    top = torch.where(some, tokens[:, 0], top)
    wide[torch.arange(rows, device="cuda"), top] = (sharp.flatten() * 6.0).to(wide.dtype)
    return wide[:, :vocab], tokens.int()


def _tokens(case, seed):
    """Keys and values of all tokens, sequence after sequence, and the new rows' queries.  Keys have channels that stand out, as a
    rotary or biased projection gives them; values have none; queries make the scores spread by a few units."""
    g = _gen(seed)
    lens, rows = _lengths(case)
    total, hkv, d = sum(lens), case["hkv"], case["d"]
    spread = torch.exp(0.4 * torch.randn(hkv, d, generator=g, device="cuda"))
    shift = 3.0 * torch.randn(hkv, d, generator=g, device="cuda") * (torch.rand(hkv, d, generator=g, device="cuda") < 0.06)
    K = torch.empty(total, hkv, d, device="cuda", dtype=_dtype(case))
    V = torch.empty(total, hkv, d, device="cuda", dtype=_dtype(case))
    for t in range(0, total, 65536):
        n = min(65536, total - t)
        K[t:t + n] = torch.randn(n, hkv, d, generator=g, device="cuda") * spread + shift
        V[t:t + n] = 0.7 * torch.randn(n, hkv, d, generator=g, device="cuda")
    Q = (1.4 * torch.randn(sum(rows), case["hq"], d, generator=g, device="cuda")).to(_dtype(case))
    return K, V, Q


def _starts(rows):
    return torch.tensor([0] + torch.tensor(rows).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


def _tree_words(case):
    """[rows, words] int64: bit u % 64 of word u / 64 says that the row sees row u of its sequence."""
    words, flat = _words(case), []
    for parents in _trees(case):
        for bits in _ancestors(parents):
            for w in range(words):
                x = bits >> (64 * w) & (2 ** 64 - 1)
                flat.append(x - 2 ** 64 if x >> 63 else x)
    return torch.tensor(flat, dtype=torch.int64, device="cuda").view(-1, words)


def prepare(case, seed):
    if case["kind"] == "logp":
        logits, tokens = _logits(case, seed)
        state = {"case": case, "logits": logits, "tokens": tokens}
        if own:
            import paper_2507_04453_amd as essa
            rows = case["rows"]
            state.update(essa=essa, ctx=essa.Context(0), logp=torch.empty(rows, case["given"], device="cuda"), entropy=torch.empty(rows, device="cuda"),
                         ids=torch.empty(rows, case["top"], dtype=torch.int32, device="cuda"), top=torch.empty(rows, case["top"], device="cuda"))
        return state
    return _prepare_accept(case, seed) if case["kind"] == "accept" else _prepare_attend(case, seed)


def _prepare_attend(case, seed):
    lens, rows = _lengths(case)
    K, V, Q = _tokens(case, seed)
    state = {"case": case, "Q": Q, "tree": _tree_words(case) if case["kind"] == "tree" else None}
    if not own:
        state["K"], state["V"], state["groups"] = _pack_plain(K), _pack_plain(V), _groups(case)
        return state
    import paper_2507_04453_amd as essa
    ctx = essa.Context(0)
    n = len(lens)
    kv = essa.KvCache(ctx, layers=1, n_kv_heads=case["hkv"], head_dim=case["d"], n_pages=sum(-(-x // case["page"]) for x in lens) + 1, page_tokens=case["page"], max_seqs=n,
                      max_tokens=max(lens))
    seqs = torch.arange(n, dtype=torch.int32, device="cuda")
    # the history comes in two turns, so that the pages of different sequences lie among one another
    at = torch.tensor([0] + lens).cumsum(0)[:-1].tolist()
    done = [0] * n
    for turn in range(2):
        upto = [length // 2 if turn == 0 else length for length in lens]
        new = [u - s for u, s in zip(upto, done)]
        index = torch.cat([torch.arange(a + s, a + u) for a, s, u in zip(at, done, upto)]).cuda()
        essa.essa_kv_extend(ctx, kv, seqs, torch.tensor(new, dtype=torch.int32, device="cuda"))
        if len(index):
            essa.essa_kv_append(ctx, kv, 0, K[index], V[index], essa.KvBatch(seqs, _starts(new), len(index)))
        done = upto
    single = case["kind"] == "sinks" and all(r == 1 for r in rows)
    state.update(essa=essa, ctx=ctx, kv=kv, scale=1.0 / math.sqrt(case["d"]), Y=torch.empty_like(Q), batch=essa.KvBatch(seqs, None if single else _starts(rows), sum(rows)))
    return state


def _groups(case):
    """Sequences of like size go through a plain pass together, padded to the longest: (their numbers, first rows, first tokens, lengths, rows) and
    the padded sizes (rows, tokens that any row sees)."""
    lens, rows = _lengths(case)
    trees = [_ancestors(p) for p in _trees(case)] if case["kind"] == "tree" else [None] * len(lens)
    toks = [_visible(case, n, r, t)[1] for n, r, t in zip(lens, rows, trees)]
    row0, tok0 = torch.tensor([0] + rows).cumsum(0).tolist(), torch.tensor([0] + lens).cumsum(0).tolist()
    groups, part = [], []
    for s in sorted(range(len(lens)), key=lambda s: (toks[s], rows[s])):
        more = part + [s]
        if part and len(more) * max(rows[i] * case["hq"] + 4 * case["hkv"] * case["d"] for i in more) * max(toks[i] for i in more) > 1e9:
            groups.append(part)
            more = [s]
        part = more
    groups.append(part)
    dev = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
    return [{"row0": dev([row0[s] for s in g]), "tok0": dev([tok0[s] for s in g]), "len": dev([lens[s] for s in g]), "rows": dev([rows[s] for s in g]),
             "R": max(rows[s] for s in g), "T": max(toks[s] for s in g)} for g in groups]


def _prepare_accept(case, seed):
    """Sequences with their drafted rows' pages handed out, the drafted rows' keys and values of every layer, and for each sequence a path from
    the root of its tree: the rows of the path, in order, in front of the sequence's part of `path`, and how many they are."""
    lens, rows = _lengths(case)
    rng = random.Random(seed)
    g = _gen(seed)
    R, n, shape = sum(rows), len(lens), (case["layers"], sum(rows), case["hkv"], case["d"])
    K = torch.randn(shape, generator=g, device="cuda").to(_dtype(case))
    V = (0.7 * torch.randn(shape, generator=g, device="cuda")).to(_dtype(case))
    path, keep = [], []
    for walk, r in zip(_paths(case), rows):
        path += walk + [0] * (r - len(walk))
        keep.append(len(walk))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    pages = [-(-x // case["page"]) for x in lens]
    n_pages, max_pages = sum(pages) + 2, max(pages)
    order = rng.sample(range(n_pages), sum(pages))
    table = torch.full((n, max_pages), -1, dtype=torch.int32)
    at = 0
    for s, k in enumerate(pages):
        table[s, :k] = torch.tensor(order[at:at + k], dtype=torch.int32)
        at += k
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[torch.tensor(order, dtype=torch.int64)] = 1
    start = table.cuda(), i32(lens), refs.cuda()
    state = {"case": case, "K": K, "V": V, "path": i32(path), "keep": i32(keep), "kept": sum(keep), "row_start": _starts(rows), "start": start}
    if own:
        import paper_2507_04453_amd as essa
        ctx = essa.Context(0)
        kv = essa.KvCache(ctx, layers=case["layers"], n_kv_heads=case["hkv"], head_dim=case["d"], n_pages=n_pages, page_tokens=case["page"], max_seqs=n, max_tokens=max(lens))
        seqs = torch.arange(n, dtype=torch.int32, device="cuda")
        back = torch.empty(2, case["layers"], sum(keep), case["hkv"], case["d"], dtype=K.dtype, device="cuda")
        state.update(essa=essa, ctx=ctx, kv=kv, back=back, served=torch.empty_like(seqs), batch=essa.KvBatch(seqs, state["row_start"], R),
                     kept_rows=essa.KvBatch(seqs, _starts(keep), sum(keep)))
    else:
        state["now"] = tuple(t.clone() for t in start)
    return state


# ---------------------------------------------------------------------------------------------- passes
def run(state):
    return _RUN[state["case"]["kind"]](state)


def _run_logp(state):
    case = state["case"]
    if own:
        state["essa"].essa_token_logprobs(state["ctx"], state["logits"], state["tokens"], state["logp"], scale=case["scale"], entropy=state["entropy"],
                                          top_ids=state["ids"] if case["top"] else None, top_logp=state["top"] if case["top"] else None)
        return {k: state[k] for k in ("logp", "entropy") + (("ids", "top") if case["top"] else ())}
    return _logp_plain(state)


def _run_attend(state):
    case = state["case"]
    if own:
        state["essa"].essa_kv_attention(state["ctx"], state["kv"], 0, state["Q"], state["Y"], state["batch"], state["scale"], window=case["window"], sinks=case["sinks"],
                                        tree=state["tree"])
        return state["Y"]
    return _attend_plain(state)


def _run_accept(state):
    # a step's trees start from the same sequences every time
    if own:
        essa, ctx, kv = state["essa"], state["ctx"], state["kv"]
        for now, start in zip((kv.table, kv.len, kv.refs), state["start"]):
            now.copy_(start)
        for layer in range(state["case"]["layers"]):
            essa.essa_kv_append(ctx, kv, layer, state["K"][layer], state["V"][layer], state["batch"])
        essa.essa_kv_accept(ctx, kv, state["batch"], state["path"], state["keep"], served=state["served"])
        for layer in range(state["case"]["layers"]):
            essa.essa_kv_read(ctx, kv, layer, state["back"][0, layer], state["back"][1, layer], state["kept_rows"])
        return state["back"], kv.table, kv.len, kv.refs, state["served"]
    return _accept_plain(state)


_RUN = {"logp": _run_logp, "sinks": _run_attend, "tree": _run_attend, "accept": _run_accept}


# ---------------------------------------------------------------------------------------------- plain forms
def _logp_plain(state):
    case, logits, tokens = state["case"], state["logits"], state["tokens"].long()
    z = logits.float() * case["scale"]
    z -= z.amax(1, keepdim=True)
    p = torch.exp(z)
    total = p.sum(1, keepdim=True)
    log_total = torch.log(total)
    out = {"logp": torch.gather(z, 1, tokens) - log_total}
    out["entropy"] = (log_total - (p * torch.where(p > 0, z, torch.zeros_like(z))).sum(1, keepdim=True) / total).flatten()
    if case["top"]:
        # larger logits first, the lower token of equal ones: whole numbers that are ordered so
        bits = (logits.float() + 0.0).view(torch.int32)        # (-0 is 0)
        bits = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
        key = (bits << 32) - torch.arange(case["vocab"], device="cuda")
        best = key.topk(case["top"], 1).values
        ids = torch.remainder(-best, 1 << 32)
        out["ids"], out["top"] = ids.int(), torch.gather(z, 1, ids) - log_total
    return out


def _pack_plain(x):
    """[tokens, heads, d] -> codes (8 bits each), scales and middles."""
    g = x.float().clamp(-32768.0, 32768.0).unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    s = ((hi - lo) * torch.full((), 1.0 / 15.0, device=x.device)).half().float()
    m = (lo + 8.0 * s).half().float()
    inverse = torch.where(s > 0, 1.0 / s, torch.zeros_like(s))
    codes = torch.round((g - m) * inverse).clamp(-8.0, 7.0).to(torch.int8).flatten(-2)
    return codes, s.squeeze(-1).half(), m.squeeze(-1).half()


def _unpack_plain(codes, s, m):
    return (m.float().unsqueeze(-1) + s.float().unsqueeze(-1) * codes.unflatten(-1, (-1, GROUP)).float()).flatten(-2)


def _attend_plain(state):
    case, Q, tree = state["case"], state["Q"], state["tree"]
    hkv, d, window, sinks = case["hkv"], case["d"], case["window"], case["sinks"]
    ratio = case["hq"] // hkv
    out = torch.empty(Q.shape, device="cuda", dtype=torch.float32)
    for g in state["groups"]:
        n, R, T = len(g["len"]), g["R"], g["T"]
        j = torch.arange(R, device="cuda")
        real = j[None, :] < g["rows"][:, None]
        row = (g["row0"][:, None] + j[None, :]).clamp(max=len(Q) - 1)
        length, base = g["len"][:, None], (g["len"] - g["rows"])[:, None]
        # the tokens that any row sees: the last T - sinks of the sequence behind its first ones, or the last T
        i = torch.arange(T, device="cuda")[None, :]
        front = torch.where(length > T, torch.full_like(length, sinks), torch.zeros_like(length))
        t = torch.where(i < front, i.expand(n, T), i + (length - T).clamp(min=0))
        inside = t < length
        at = (g["tok0"][:, None] + t).clamp(max=state["K"][0].shape[0] - 1)
        if tree is None:
            pos = base + j[None, :]
            seen = t[:, None, :] <= pos[:, :, None]
        else:
            u = t - base                                       # which of the tree's rows a token is
            word = (u.clamp(min=0) // 64).clamp(max=tree.shape[1] - 1)
            bits = torch.gather(tree[row], 2, word[:, None, :].expand(n, R, T)) >> (u.clamp(min=0) % 64)[:, None, :] & 1
            drafted = (u >= 0)[:, None, :]
            mine = (drafted & (bits > 0)) & inside[:, None, :]
            pos = base + mine.sum(2) - 1
            seen = mine | ~drafted
        if window:
            near = (t[:, None, :] > (pos - window)[:, :, None]) | (t < sinks)[:, None, :]
            seen = seen & near if tree is None else seen & (near | drafted)
        seen = seen & inside[:, None, :]
        k, v = (_unpack_plain(*(x[at] for x in state[name])).transpose(1, 2) for name in ("K", "V"))               # [n, hkv, T, d]
        q = Q[row].float().view(n, R, hkv, ratio, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, ratio * R, d)
        scores = (torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))).view(n, hkv, ratio, R, T)
        scores.masked_fill_(~seen[:, None, None], float("-inf"))
        scores = torch.exp(scores - scores.amax(4, keepdim=True).clamp(min=-3e38))
        o = torch.matmul(scores.view(n, hkv, ratio * R, T), v.contiguous()).view(n, hkv, ratio, R, d) / scores.sum(4, keepdim=True)
        o = o.permute(0, 3, 1, 2, 4).reshape(n, R, hkv * ratio, d)
        out[row[real]] = o[real]
    return out.to(Q.dtype)


def _accept_plain(state):
    case = state["case"]
    table, length, refs = state["now"]
    for now, start in zip(state["now"], state["start"]):
        now.copy_(start)
    n, R, kept, keep = len(length), state["K"].shape[1], state["kept"], state["keep"].long()
    first = state["row_start"].long()
    packed = [_pack_plain(x) for x in (state["K"], state["V"])]
    # kept row i of the call is row `source` of the drafted ones
    to = torch.cumsum(keep, 0)
    which = torch.arange(kept, device="cuda")
    seq = torch.searchsorted(to, which, right=True)
    at = first[seq] + which - (to - keep)[seq]
    source = first[seq] + state["path"].long()[at]
    back = torch.stack([_unpack_plain(*(x[:, source] for x in p)).to(state["K"].dtype) for p in packed])
    # what lies behind the kept rows goes back
    page = case["page"]
    before = -(-length.long() // page)
    length.copy_((length - (first[1:] - first[:-1]) + keep).int())
    after = -(-length.long() // page)
    column = torch.arange(table.shape[1], device="cuda")[None, :]
    gone = (column >= after[:, None]) & (column < before[:, None])
    refs.index_add_(0, table[gone].long(), -torch.ones_like(table[gone]))
    table[gone] = -1
    return back, table, length, refs, torch.arange(n, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------------------------- 64 bits
def _single(x):
    """What one operation in single precision gives: the result in 64 bits, rounded once."""
    return x.float().double()


def _levels_exact(x):
    """The values that rows stand for in the cache, in 64 bits; x: [..., d]."""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    r = float(torch.tensor(1.0 / 15.0, dtype=torch.float32))
    for c in range(0, x.shape[-1], GROUP):
        v = torch.clip(x[..., c:c + GROUP].double(), -32768.0, 32768.0)
        low = torch.min(v, -1, keepdim=True).values
        high = torch.max(v, -1, keepdim=True).values
        s = _single(_single(high - low) * r).half().double()
        m = _single(low + 8 * s).half().double()
        q = torch.round(_single(_single(v - m) * _single(1 / torch.where(s == 0, torch.ones_like(s), s))))
        q = torch.where(s == 0, torch.zeros_like(q), torch.clip(q, -8, 7))
        out[..., c:c + GROUP] = m + s * q
    return out


def exact(case, seed):
    return {"logp": _exact_logp, "sinks": _exact_attend, "tree": _exact_attend, "accept": _exact_accept}[case["kind"]](case, seed)


def _exact_logp(case, seed):
    logits, tokens = _logits(case, seed)
    scale = float(torch.tensor(case["scale"], dtype=torch.float32))
    parts = []
    for i in range(0, case["rows"], 256):
        x = logits[i:i + 256].double() * scale
        lse = torch.logsumexp(x, 1, keepdim=True)
        logp = x - lse
        entropy = torch.special.entr(torch.exp(logp)).sum(1)
        part = [torch.take_along_dim(logp, tokens[i:i + 256].long(), 1), entropy]
        if case["top"]:
            part.append(torch.sort(logp, 1, descending=True).values[:, :case["top"]])
        parts.append(part)
    out = [torch.cat(p) for p in zip(*parts)]
    return {"logp": out[0], "entropy": out[1], **({"ids": None, "top": out[2]} if case["top"] else {})}


def _exact_attend(case, seed):
    if work(case)["flops"] > 3e12:
        return None
    lens, rows = _lengths(case)
    K, V, Q = _tokens(case, seed)
    ratio, out = case["hq"] // case["hkv"], torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    trees = _trees(case) if case["kind"] == "tree" else None
    at = row = 0
    for s, (length, new) in enumerate(zip(lens, rows)):
        k, v = _levels_exact(K[at:at + length]), _levels_exact(V[at:at + length])
        for j in range(0, new, 512):
            n = min(512, new - j)
            last = torch.arange(length - new + j, length - new + j + n, device="cuda").view(n, 1)
            t = torch.arange(length, device="cuda").view(1, length)
            if trees is None:
                seen = t <= last
                if case["window"]:
                    seen = seen & ((last - t < case["window"]) | (t < case["sinks"]))
            else:
                line = torch.zeros(n, new, dtype=torch.bool)
                for i in range(n):
                    up = j + i
                    while up >= 0:
                        line[i, up] = True
                        up = trees[s][up]
                line = line.cuda()
                depth = line.sum(1, keepdim=True) - 1
                seen = torch.ones(n, length, dtype=torch.bool, device="cuda")
                if case["window"]:
                    seen = (length - new + depth - t < case["window"]) | (t < case["sinks"])
                seen[:, length - new:] = line
            for h in range(case["hq"]):
                z = torch.mm(Q[row + j:row + j + n, h].double(), k[:, h // ratio].t().contiguous()) / math.sqrt(case["d"])
                out[row + j:row + j + n, h] = torch.mm(torch.softmax(z.masked_fill(~seen, -math.inf), 1), v[:, h // ratio].contiguous())
        at += length
        row += new
    return out


def _exact_accept(case, seed):
    state = _prepare_accept(case, seed)
    source, first = [], state["row_start"].tolist()
    path = state["path"].tolist()
    for s, n in enumerate(state["keep"].tolist()):
        source += [first[s] + path[first[s] + i] for i in range(n)]
    rows = torch.tensor(source, dtype=torch.int64, device="cuda")
    return torch.stack([_levels_exact(x[:, rows]) for x in (state["K"], state["V"])]), None, None, None, None
