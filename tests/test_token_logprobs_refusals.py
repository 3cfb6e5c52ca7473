"""What essa_token_logprobs refuses, found on the host before anything is launched; and the oracle's own numbers."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle as orc
import paper_2507_04453_amd as essa

GOOD = dict(ctx=True, logits=256, stride=100, x_dtype=0, R=3, V=100, scale=1.0, tokens=256, n_tokens=2, logp=256, entropy=256, n_top=4, top_ids=256, top_logp=256)


def _call(**change):
    """Pointers are numbers that nothing reads: every call here is refused, or has no rows."""
    a = {**GOOD, **change}
    blank = C.create_string_buffer(4096)                       # a context that nobody made; refusals come before it is looked at
    names = ("logits", "stride", "x_dtype", "R", "V", "scale", "tokens", "n_tokens", "logp", "entropy", "n_top", "top_ids", "top_logp")
    code = essa.lib.essa_token_logprobs(C.cast(blank, C.c_void_p) if a["ctx"] else None, *[a[n] for n in names])
    return code, essa.lib.essa_last_error().decode()


@pytest.mark.parametrize("change,code", [
    (dict(ctx=False), 1), (dict(x_dtype=2), 1), (dict(x_dtype=-1), 1), (dict(R=-1), 2), (dict(R=2 ** 24 + 1), 2), (dict(V=0), 2), (dict(V=2 ** 28 + 1, stride=2 ** 29), 2),
    (dict(stride=99), 2), (dict(stride=-100), 2), (dict(stride=2 ** 32 + 1), 2), (dict(n_tokens=-1), 2), (dict(n_tokens=4097), 2), (dict(n_top=-1), 2), (dict(n_top=65), 2),
    (dict(V=2 ** 19 + 1, stride=2 ** 20), 3), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(scale=3e38), 1),
    (dict(logits=None), 1), (dict(tokens=None), 1), (dict(logp=None), 1), (dict(top_ids=None), 1), (dict(top_logp=None), 1), (dict(logits=258), 1), (dict(logits=257, x_dtype=1), 1),
])
def test_refused(change, code):
    got, text = _call(**change)
    assert got == code, (got, text)
    assert "essa_token_logprobs" in text


def test_no_rows_is_nothing_to_do():
    assert _call(R=0, logits=None, tokens=None)[0] == 0


@pytest.mark.parametrize("shapes", [
    dict(logits=(3, 4, 5)), dict(tokens=(2,)), dict(tokens=(3, 2), logp=(3, 1)), dict(tokens=(3,), logp=None), dict(entropy=(3, 1)), dict(entropy=(2,)),
    dict(top_ids=(3, 2), top_logp=(3, 3)), dict(top_ids=(2, 2), top_logp=(2, 2)), dict(top_ids=(3, 2)),
])
def test_shapes_that_do_not_fit(shapes):
    meta = {k: None if s is None else torch.empty(s, device="meta", dtype=torch.int32 if k in ("tokens", "top_ids") else torch.float32) for k, s in shapes.items()}
    logits = meta.pop("logits", torch.empty(3, 9, device="meta"))
    logits.__class__ = type("OnGpu", (torch.Tensor,), {"is_cuda": True})
    if "tokens" in meta and "logp" not in meta:
        meta["logp"] = torch.empty(meta["tokens"].shape, device="meta")
    with pytest.raises(ValueError):
        essa.essa_token_logprobs(None, logits, **meta)


def test_oracle():
    """Closed forms: equal logits, one certain token, and log probabilities that sum to one."""
    x = np.zeros((3, 8))
    x[1, 3] = 1e4
    x[2] = np.log(np.arange(1, 9))
    lp, h, ids, top = orc.token_logprobs(x, [[0, 7], [3, -1], [7, 8]], n_top=3)
    assert np.allclose(lp[0], -np.log(8)) and np.isclose(h[0], np.log(8)) and ids[0].tolist() == [0, 1, 2]
    assert lp[1].tolist() == [0.0, 0.0] and h[1] == 0 and ids[1].tolist() == [3, 0, 1]
    p = np.arange(1, 9) / 36
    assert np.isclose(lp[2, 0], np.log(8 / 36)) and np.isnan(lp[2, 1]) and np.isclose(h[2], -(p * np.log(p)).sum()) and ids[2].tolist() == [7, 6, 5]
    assert np.allclose(top[2], np.log(p[::-1][:3]))
    lp, h, ids, top = orc.token_logprobs(np.full((1, 4), -np.inf), [[0]], n_top=2)
    assert lp[0, 0] == -np.inf and h[0] == 0 and (ids == -1).all() and (top == -np.inf).all()
