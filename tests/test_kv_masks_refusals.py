"""What attention with masks and the keeping of a path refuse, found on the host before anything is launched; masks and paths of the oracle."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle as orc
import paper_2507_04453_amd as essa
from kv_masks import ancestors
from paper_2507_04453_amd import essa as binding


class _Cache(C.Structure):
    """The head of a cache object, as the checks look at it: no device memory behind it, and none is looked at by calls that are refused."""
    _fields_ = [("ctx", C.c_void_p), ("device", C.c_int), ("d", binding._KvDesc), ("rest", C.c_char * 256)]


def _objects():
    blank = C.create_string_buffer(4096)
    ctx = C.cast(blank, C.c_void_p)
    kv = _Cache(ctx.value, 0, binding._KvDesc(2, 4, 64, 64, 8, 6, 4, 256, 256, 256, 256))
    return blank, ctx, kv


def _attend(layer=0, stride=512, dtype=1, heads=8, R=3, n=3, window=0, sinks=0, tree=256, words=1, scale=0.1, mask=True, kv_of_another=False, q=256, y=256):
    keep, ctx, kv = _objects()
    if kv_of_another:
        kv.ctx = 1
    batch = binding._KvBatch(256, 256, n, R)
    m = binding._KvMask(window, sinks, tree, words)
    code = essa.lib.essa_kv_attention_masked(ctx, C.byref(kv), layer, q, stride, dtype, heads, C.byref(batch), scale, C.byref(m) if mask else None, y, stride, dtype)
    return code, essa.lib.essa_last_error().decode()


@pytest.mark.parametrize("change,code", [
    (dict(mask=False), 1), (dict(window=-1), 1), (dict(sinks=-1), 1), (dict(words=-1), 2), (dict(words=17), 2), (dict(tree=None), 1), (dict(tree=260), 1), (dict(layer=2), 2),
    (dict(layer=-1), 2), (dict(heads=6), 2), (dict(heads=0), 2), (dict(dtype=7), 1), (dict(stride=511), 2), (dict(R=-1), 2), (dict(R=2 ** 24 + 1), 2), (dict(n=7), 2), (dict(n=0), 2),
    (dict(scale=float("nan")), 1), (dict(scale=3e38), 1), (dict(kv_of_another=True), 6), (dict(q=None), 1), (dict(y=None), 1), (dict(q=257), 1),
])
def test_attention_refused(change, code):
    got, text = _attend(**change)
    assert got == code, (got, text)
    assert "essa_kv_attention_masked" in text


def test_no_rows_is_nothing_to_do():
    assert _attend(R=0, tree=None)[0] == 0 and _attend(R=0, words=0, tree=3)[0] == 0


@pytest.mark.parametrize("change,code", [(dict(path=None), 1), (dict(keep=None), 1), (dict(n=7), 2), (dict(R=-1), 2), (dict(another=True), 6), (dict(batch=False), 1)])
def test_accept_refused(change, code):
    a = {**dict(path=256, keep=256, n=3, R=9, another=False, batch=True), **change}
    blank, ctx, kv = _objects()
    if a["another"]:
        kv.ctx = 1
    batch = binding._KvBatch(256, 256, a["n"], a["R"])
    got = essa.lib.essa_kv_accept(ctx, C.byref(kv), C.byref(batch) if a["batch"] else None, a["path"], a["keep"], None)
    assert got == code and "essa_kv_accept" in essa.lib.essa_last_error().decode()
    assert essa.lib.essa_kv_accept(ctx, C.byref(kv), C.byref(binding._KvBatch(None, None, 0, 0)), None, None, None) in (0, 6)


def test_python_checks():
    fake = type("Fake", (), {"n": 2, "R": 5, "ref": None})
    kv = type("Kv", (), {"head_dim": 64, "n_kv_heads": 2, "_h": None})
    on = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, device="meta", dtype=dtype).as_subclass(type("OnGpu", (torch.Tensor,), {"is_cuda": True, "data_ptr": lambda s: 256}))
    with pytest.raises(ValueError):
        essa.essa_kv_accept(None, kv, fake, on(4, dtype=torch.int32), on(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        essa.essa_kv_accept(None, kv, fake, on(5, dtype=torch.int32), on(3, dtype=torch.int32))
    q = on(5, 2, 64)
    for tree in (on(4, 1, dtype=torch.int64), on(5, 0, dtype=torch.int64), on(5, 1, 1, dtype=torch.int64)):
        with pytest.raises(ValueError):
            essa.essa_kv_attention(None, kv, 0, q, q, fake, 0.1, tree=tree)
    with pytest.raises(ValueError):
        essa.essa_kv_attention(None, kv, 0, q, q, fake, 0.1, causal=False, sinks=3)


def test_masks_of_the_oracle():
    """By brute force from the definition, one pair at a time."""
    g = np.random.default_rng(0)
    for _ in range(200):
        L, rows, window, sinks = int(g.integers(0, 12)), int(g.integers(1, 9)), int(g.integers(0, 6)), int(g.integers(0, 5))
        seen, base = orc.kv_mask(L, rows, window, sinks), L - rows
        for j in range(rows):
            for t in range(L):
                p = base + j
                assert seen[j, t] == (t <= p and (window == 0 or t > p - window or t < sinks))
        tree = g.random((rows, rows)) < 0.4
        seen = orc.kv_mask(L, rows, window, sinks, tree)
        for j in range(rows):
            p = base + sum(bool(tree[j, u]) for u in range(rows) if u != j and base + u >= 0)
            for t in range(L):
                if t >= base:
                    assert seen[j, t] == tree[j, t - base]
                else:
                    assert seen[j, t] == (window == 0 or t > p - window or t < sinks)
    parents = [-1, 0, 0, 2, -1, 4]
    assert ancestors(parents).astype(int).tolist() == [[1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 0, 1, 0, 0, 0], [1, 0, 1, 1, 0, 0], [0, 0, 0, 0, 1, 0], [0, 0, 0, 0, 1, 1]]


def test_paths_of_the_oracle():
    m = orc.KvPages(8, 4, 3, 4)
    m.extend([0, 1], [list("abcdefg"), list("hij")])
    m.fork([0], [2], [4])
    assert m.accept([0, 1, -1], [3, 2, 1], [[0, 2], [1], []], [2, 1, 0]) == [0, 1, orc.KV_SKIPPED]
    assert m.tokens[0] == list("abcdeg") and m.tokens[1] == list("hj")
    assert m.accept([0, 0, 1, 1], [2, 2, 2, 1], [[1, 0], [0], [0, 0], []], [2, 1, 2, 2]) == [orc.KV_BAD_ENTRY] * 4
    assert m.accept([0], [6], [[]], [0]) == [orc.KV_BAD_ENTRY]            # its first page is the fork's too
    assert m.accept([0], [2], [[]], [0]) == [0] and len(m.pages[0]) == 1 and sum(r > 0 for r in m.refs) == 2
