"""Log probabilities of given tokens, entropies and the most probable tokens, element by element against 64 bits, with the bounds that the
sums' arithmetic gives (oracle.token_logprobs_limits); tokens and their order exactly."""
import numpy as np
import pytest
import torch

import oracle as orc
from kv_helpers import host, i32, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(essa):
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    c = essa.Context(0)
    yield c
    c.close()


DTYPES = [torch.bfloat16, torch.float32]


def _logits(R, V, dtype, seed, spread=2.0, edit=None, pad=0, shift=0):
    """(64-bit numpy, GPU view [R, V] whose rows lie V + pad apart, `shift` values behind the beginning of memory; NaN around them)."""
    x = values((R, V), np.random.default_rng(seed), torch.float32, scale=spread)[0]
    if edit:
        edit(x)
    flat = torch.full((R * (V + pad) + shift + 8,), float("nan"), device="cuda", dtype=dtype)
    view = flat[shift:shift + R * (V + pad)].view(R, V + pad)[:, :V]
    view.copy_(torch.from_numpy(x))
    return host(view.contiguous()), view


def _check(essa, ctx, x, view, tokens, n_top, scale=1.0, entropy=True):
    R, V = x.shape
    print("logprobs R=%d V=%d %s tokens=%s top=%d scale=%g stride=%d" % (R, V, view.dtype, None if tokens is None else tokens.shape, n_top, scale, view.stride(0)), flush=True)
    t = None if tokens is None else torch.from_numpy(tokens.astype(np.int32)).cuda()
    guard = lambda shape, dtype=torch.float32: torch.full((int(np.prod(shape)) + 16,), 77, device="cuda", dtype=dtype)
    cut = lambda g, shape: g[8:8 + int(np.prod(shape))].view(shape)
    shapes = {"logp": None if t is None else tuple(t.shape), "entropy": (R,) if entropy else None, "top_ids": (R, n_top) if n_top else None, "top_logp": (R, n_top) if n_top else None}
    mem = {k: guard(s, torch.int32 if k == "top_ids" else torch.float32) for k, s in shapes.items() if s is not None}
    out = {k: cut(mem[k], s) if s is not None else None for k, s in shapes.items()}
    essa.essa_token_logprobs(ctx, view, t, out["logp"], scale, out["entropy"], out["top_ids"], out["top_logp"])
    for k, m in mem.items():
        m = m.cpu()
        assert (m[:8] == 77).all() and (m[-8:] == 77).all(), ("written outside of", k)
    scale = float(np.float32(scale))
    lp, h, ids, top = orc.token_logprobs(x, np.zeros((R, 0)) if tokens is None else tokens, scale, n_top)
    a, b = orc.token_logprobs_limits(x, scale)

    def close(got, want, limit, what):
        got = got.reshape(want.shape)
        want = np.where(np.abs(want) > np.finfo(np.float32).max, np.sign(want) * np.inf, want)         # outputs are fp32: what it does not hold is an infinity
        same = (np.isnan(got) & np.isnan(want)) | (got == want)
        with np.errstate(invalid="ignore"):
            ok = same | (np.abs(got - want) <= limit)
        assert ok.all(), (what, np.argwhere(~ok)[0], got[~ok][0], want[~ok][0], np.broadcast_to(limit, want.shape)[~ok][0])
    with np.errstate(invalid="ignore"):
        if t is not None:
            close(host(out["logp"]), lp, a[:, None] + 2.0 ** -21 * np.abs(np.where(np.isfinite(lp), lp, 0)), "logp")
        if entropy:
            close(host(out["entropy"]), h, b, "entropy")
        if n_top:
            got = out["top_ids"].cpu().numpy()
            assert np.array_equal(got, ids), ("top ids", np.argwhere(got != ids)[0], got[got != ids][0], ids[got != ids][0])
            close(host(out["top_logp"]), top, a[:, None] + 2.0 ** -21 * np.abs(np.where(np.isfinite(top), top, 0)), "top")
    return out


def _tokens(R, V, n, seed):
    return np.random.default_rng(seed).integers(0, V, (R, n))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V,n,top", [
    (1, 1, 1, 1), (3, 2, 2, 64), (2, 7, 1, 5), (5, 64, 3, 3), (1, 65, 1, 64), (4, 511, 1, 8), (2, 512, 1, 0), (3, 513, 2, 20), (1, 4095, 1, 5), (7, 4097, 16, 1),
    (2, 32001, 4, 64), (1, 152064, 1, 5), (300, 1000, 1, 3), (40, 20011, 2, 20), (600, 515, 1, 7), (1, 524288, 1, 2), (4, 511, 1, 64), (3, 513, 1, 63), (600, 900, 1, 64), (2, 4000, 1, 64), (2, 8200, 1, 64),
    (3, 8192, 1, 33), (2, 300001, 1, 40), (600, 8001, 1, 32), (200, 5000, 1, 9), (256, 20011, 1, 64), (193, 70001, 2, 5), (520, 66000, 1, 5), (515, 4100, 1, 64), (257, 9000, 1, 3),
])
def test_sizes(essa, ctx, dtype, R, V, n, top):
    x, view = _logits(R, V, dtype, 1)
    _check(essa, ctx, x, view, _tokens(R, V, n, 2), top)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 8), (13, 7)])
@pytest.mark.parametrize("R,V", [(5, 1000), (3, 8), (2, 9001)])
def test_rows_anywhere(essa, ctx, dtype, pad, shift, R, V):
    """Memory around the rows holds NaN."""
    x, view = _logits(R, V, dtype, 3, pad=pad, shift=shift)
    _check(essa, ctx, x, view, _tokens(R, V, 2, 4), 6)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [0.1, 1 / 0.7, 3.0, 1e-30])
def test_temperatures(essa, ctx, dtype, scale):
    x, view = _logits(6, 5000, dtype, 5)
    _check(essa, ctx, x, view, _tokens(6, 5000, 3, 6), 10, scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [2, 520, 200])
def test_sharp_and_flat_rows(essa, ctx, dtype, R):
    """One certain token, equal logits, logits far from zero, rising ones (every lane's maximum moves all the time)."""
    def edit(x):
        V = x.shape[1]
        x[0] = np.linspace(-300, 300, V)
        x[1::5] = 0
        x[2::5, 17] = 200
        x[3::5] += 1000
        x[4::5] -= 1000
    x, view = _logits(R, 9000, dtype, 7, edit=edit)
    _check(essa, ctx, x, view, _tokens(R, 9000, 2, 8), 12)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", [(5, 3000), (3, 60000), (200, 9000), (520, 9000)])
def test_tokens_that_are_all_but_certain(essa, ctx, dtype, R, V):
    """The log probability of a token far ahead of all others, and the entropy of its row, to the last bits of themselves: with G the exponents of 2 that others
    are behind (those that count), a weight is off by 6 G u at most (its exponent's rounding and twice its factor's), their sum by V / 256 + 20 more, what
    is made of it by 8 u."""
    g = np.random.default_rng(40)
    at = g.integers(0, V, R)
    lead = np.where(np.arange(R) % 3 == 0, 12.0, np.where(np.arange(R) % 3 == 1, 20.0, 30.0))

    def edit(x):
        x[np.arange(R), at] = 9.0 + lead
    x, view = _logits(R, V, dtype, 41, edit=edit)
    out = _check(essa, ctx, x, view, np.stack([at, (at + 1) % V], 1), 2)
    z = x - x.max(1, keepdims=True)
    z[np.arange(R), at] = -np.inf
    rest = np.exp(z).sum(1)
    G = ((x.max(1) - np.sort(x, 1)[:, -2]) + 8) / np.log(2)              # what is 8 nats behind the first of them counts for little
    far = -(np.exp(z) * np.where(np.isfinite(z), z, 0)).sum(1)
    h = np.log1p(rest) + far / (1 + rest)
    limit = (V / 256 + 28 + 6 * G) * 2.0 ** -24
    lp, got = host(out["logp"])[:, 0], host(out["entropy"])
    assert (np.abs(lp + np.log1p(rest)) <= limit * rest).all(), np.max(np.abs(lp + np.log1p(rest)) / rest / limit)
    assert (np.abs(got - h) <= 2 * limit * h).all(), np.max(np.abs(got - h) / h / limit)
    assert out["top_ids"][:, 0].tolist() == at.tolist() and np.array_equal(host(out["top_logp"])[:, 0], lp)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [3, 200, 530])
def test_two_or_more_largest_ones(essa, ctx, dtype, R):
    """The largest value several times, in one lane's load, in different lanes, waves and parts: none of them is lost or counted twice."""
    V = 9000

    def edit(x):
        for i in range(R):
            x[i, [0, 1, 700, 8999][:i % 4 + 1]] = 40.0
            if i % 5 == 0:
                x[i, 512:520] = 40.0
    x, view = _logits(R, V, dtype, 42, edit=edit)
    _check(essa, ctx, x, view, np.tile([0, 1, 5], (R, 1)), 3)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", [(4, 700), (4, 40000), (515, 3000), (515, 6000), (200, 40000), (515, 66000)])
def test_equal_logits_come_in_order(essa, ctx, dtype, R, V):
    """Few levels, so that almost everything is a tie: the lower tokens are taken, and -0 equals 0."""
    def edit(x):
        g = np.random.default_rng(9)
        x[:] = g.integers(0, 3, x.shape)
        x[0] = 0
        x[1] = np.where(g.random(x.shape[1]) < 0.5, -0.0, 0.0)
        x[2] = -5
        x[2, V // 2:V // 2 + 100] = 3                           # neighbours
        x[3] = np.sort(x[3])[::-1]
    x, view = _logits(R, V, dtype, 10, edit=edit)
    _check(essa, ctx, x, view, _tokens(R, V, 1, 11), 64)
    _check(essa, ctx, x, view, None, 5, entropy=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", [(12, 900), (12, 30000), (520, 600), (520, 6000), (200, 30000), (515, 66000)])
def test_forbidden_tokens(essa, ctx, dtype, R, V):
    """-inf: most of a row, all but a few, all of it.  The type's lowest value is a value, in part of a row or all over it."""
    low = float(torch.finfo(dtype).min)

    def edit(x):
        g = np.random.default_rng(12)
        x[g.random(x.shape) < 0.5] = -np.inf
        x[0] = -np.inf
        x[1, :] = -np.inf
        x[1, [3, V - 1]] = [1.0, 2.0]
        x[2] = low
        x[3] = low
        x[3, [5, V // 2]] = [0.5, 0.25]
        x[4] = np.where(g.random(V) < 0.5, low, -np.inf)
        x[5] = -low
        x[6] = low
        x[6, 7] = -low
        x[7] = -np.inf
        x[7, V // 3] = low
        x[8] = 3e37
        x[8, 2] = -1e38
        x[9] = -np.inf
        x[9, 0] = -2.0
    x, view = _logits(R, V, dtype, 13, edit=edit)
    with np.errstate(over="ignore"):
        for scale in (1.0, 2.0):
            out = _check(essa, ctx, x, view, np.concatenate([_tokens(R, V, 3, 14), np.tile([3, 7], (R, 1))], 1), 9, scale)
    assert out["top_ids"][0].tolist() == [-1] * 9 and out["top_ids"][1].tolist() == [V - 1, 3] + [-1] * 7 and out["top_ids"][2].tolist() == list(range(9))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", [(8, 1000), (8, 20000), (520, 600), (520, 6000), (200, 20000)])
def test_rows_that_are_not_finite(essa, ctx, dtype, R, V):
    """A NaN of either sign or a +inf anywhere makes its row NaN and no other."""
    def edit(x):
        x[0, 0] = np.nan
        x[1, V - 1] = np.nan
        x[2, V // 2] = np.inf
        x[3] = np.nan
        x[4] = -np.inf
        x[4, 5] = np.nan
        x[5, 3] = -np.float32(np.nan)
        x[6] = -3e38
        x[6, 9] = np.nan
    x, view = _logits(R, V, dtype, 15, edit=edit)
    _check(essa, ctx, x, view, _tokens(R, V, 2, 16), 4)


def test_tokens_that_are_not_there(essa, ctx):
    x, view = _logits(3, 100, torch.float32, 17)
    _check(essa, ctx, x, view, np.array([[-1, 0, 99], [100, 5, -7], [2 ** 31 - 1, -2 ** 31, 1]]), 0)


def test_what_is_not_asked_for(essa, ctx):
    x, view = _logits(3, 3001, torch.bfloat16, 18)
    _check(essa, ctx, x, view, _tokens(3, 3001, 1, 19)[:, 0], 0, entropy=False)
    _check(essa, ctx, x, view, None, 0)
    essa.essa_token_logprobs(ctx, view)
    essa.essa_token_logprobs(ctx, view[:0], torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda"))


def test_many_rows_twice(essa, ctx):
    """More rows than the chip takes at once, and the same bits again."""
    R, V = 9000, 700
    x, view = _logits(R, V, torch.bfloat16, 20)
    t = _tokens(R, V, 1, 21)
    a = _check(essa, ctx, x, view, t, 3)
    b = _check(essa, ctx, x, view, t, 3)
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_offsets_past_32_bits(essa, ctx):
    """Rows 2^30 values apart: the last begins 6 GB in."""
    V = 1000
    mem = torch.empty(3 * 2 ** 30 + V, device="cuda", dtype=torch.bfloat16)
    view = torch.as_strided(mem, (4, V), (2 ** 30, 1))
    x = values((4, V), np.random.default_rng(22), torch.bfloat16)[1]
    view.copy_(x)
    _check(essa, ctx, host(x), view, _tokens(4, V, 1, 23), 5)


def test_recorded(essa):
    """A row shared among workgroups in a recorded call, replayed with new logits, with larger and smaller eager calls of the context between."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        big, big_view = _logits(30, 60000, torch.float32, 24)
        _check(essa, ctx, big, big_view, _tokens(30, 60000, 1, 25), 9)
        R, V = 3, 50001
        logits = torch.empty(R, V, device="cuda", dtype=torch.bfloat16)
        t = _tokens(R, V, 2, 26)
        tokens, logp, h = torch.from_numpy(t).int().cuda(), torch.empty(R, 2, device="cuda"), torch.empty(R, device="cuda")
        ids, top = torch.empty(R, 6, device="cuda", dtype=torch.int32), torch.empty(R, 6, device="cuda")
        torch.cuda.synchronize()
        ctx.graph_begin()
        essa.essa_token_logprobs(ctx, logits, tokens, logp, 1.0, h, ids, top)
        graph = ctx.graph_end()
        for i in range(4):
            x, view = _logits(R, V, torch.bfloat16, 27 + i)
            logits.copy_(view)
            for out in (logp, h, ids, top):
                out.fill_(5)
            graph.launch()
            torch.cuda.synchronize()
            want = _check(essa, ctx, x, view, t, 6)
            assert torch.equal(want["logp"], logp) and torch.equal(want["entropy"], h) and torch.equal(want["top_ids"], ids) and torch.equal(want["top_logp"], top)
            _check(essa, ctx, big, big_view, _tokens(30, 60000, 1, 25), 9)
        graph.close()
        ctx.close()


def test_first_call_is_not_recorded(essa):
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = essa.Context(0, stream)
        x, view = _logits(2, 300, torch.float32, 31)
        ctx.graph_begin()
        with pytest.raises(essa.EssaError) as e:
            essa.essa_token_logprobs(ctx, view, entropy=torch.empty(2, device="cuda"))
        ctx.graph_end().close()
        assert e.value.code == 6
        _check(essa, ctx, x, view, _tokens(2, 300, 1, 32), 2)
        ctx.close()


def test_rewards_of_candidates(essa, ctx):
    """Log probabilities as rewards: every candidate's mean over its rows, and their order."""
    K, per, V = 6, 30, 4000
    x, view = _logits(K * per, V, torch.bfloat16, 33)
    t = _tokens(K * per, V, 1, 34)
    out = _check(essa, ctx, x, view, t, 0)
    F, order = torch.zeros(K, device="cuda"), torch.empty(K, dtype=torch.int32, device="cuda")
    essa.essa_reward_accumulate(ctx, out["logp"].view(-1, 1), torch.ones(1, device="cuda"), i32(np.repeat(range(K), per)), F)
    essa.essa_rank_rewards(ctx, F, order)
    lp = orc.token_logprobs(x, t)[0].reshape(K, per)
    want = lp.mean(1)
    a = orc.token_logprobs_limits(x)[0].max()
    assert np.abs(host(F) - want).max() <= a + 2.0 ** -20 * np.abs(lp).max()
    assert np.array_equal(order.cpu().numpy(), np.argsort(-host(F), kind="stable"))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [4, 530])
@pytest.mark.parametrize("scale", [2.0 ** -120, 1e-12, 1e6, 1e30, 1e36])
def test_extreme_scales(essa, ctx, dtype, R, scale):
    """From rows that are all but flat to rows whose values, times the scale, single precision does not hold."""
    x, view = _logits(R, 3001, dtype, 35)
    _check(essa, ctx, x, view, _tokens(R, 3001, 2, 36), 5, scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,V", [(26, 900), (13, 30000), (533, 600), (520, 6000), (208, 30000)])
@pytest.mark.parametrize("scale", [1.0, 0.3])
def test_values_that_stand_for_nothing(essa, ctx, dtype, R, V, scale):
    """Large numbers in forbidden places, in front of the logits that count, among them, everywhere; logits of every size, where single precision's steps of scaled
    logits are below one, a few, and far more."""
    def edit(x):
        g = np.random.default_rng(37)
        half = g.random(V) < 0.5
        for i, fill in enumerate((-1e30, -1e20, -1e9, -1e5, -6e7)):
            x[i::13, :3 * V // 4] = fill
            x[i + 5::13, half] = fill
        x[1::13] = -1e30
        x[1::13, V - 2] = 3.0
        x[5::13] = -1e30
        x[6::13] = 1e30
        x[6::13, half] = 9.9e29
        for i, shift in ((10, 1e9), (11, 4.65e7), (12, -4.65e7)):
            x[i::13] = shift + 20 * x[i::13]
    x, view = _logits(R, V, dtype, 38, edit=edit)
    tokens = np.concatenate([_tokens(R, V, 3, 39), np.full((R, 1), V - 2)], 1)
    _check(essa, ctx, x, view, tokens, 9, scale)
    _check(essa, ctx, -x, view.mul_(-1), tokens, 9, scale)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [3, 520])
def test_small_scales_of_large_logits(essa, ctx, dtype, R):
    """Differences of logits that are past all numbers, but not so times the scale."""
    def edit(x):
        x[:] = np.linspace(-1, 1, x.shape[1]) * float(torch.finfo(dtype).max)
    x, view = _logits(R, 2000, dtype, 40, edit=edit)
    _check(essa, ctx, x, view, _tokens(R, 2000, 4, 41), 6, 2.0 ** -126)
    _check(essa, ctx, x, view, _tokens(R, 2000, 4, 41), 6, 0.25)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,top", [(4100, 5), (8100, 64), (16300, 40), (16300, 64), (16383, 3), (900, 64)])
def test_many_rows_of_middle_size(essa, ctx, dtype, V, top):
    """One wave a row; equal, sorted, forbidden and all but certain logits among them."""
    def edit(x):
        g = np.random.default_rng(42)
        x[::7] = np.round(x[::7])
        x[1::70] = np.sort(x[1::70])
        x[2::70] = -np.sort(-x[2::70])
        x[3::70] = 1.0
        x[4::7][g.random(x[4::7].shape) < 0.997] = -np.inf
        x[5::7, 77] = 40.0
    x, view = _logits(2050, V, dtype, 43, edit=edit, pad=3)
    _check(essa, ctx, x, view, _tokens(2050, V, 1, 44), top)


@pytest.mark.parametrize("seed", range(24))
def test_any_call(essa, ctx, seed):
    """Sizes, strides, scales, forbidden tokens and outputs as they come."""
    g = np.random.default_rng(2000 + seed)
    V = int(np.exp(g.uniform(0, np.log(200000 if seed % 3 else 3000))))
    R = int(min(np.exp(g.uniform(0, np.log(1200))), 1 + 1.5e6 // V))
    share = float(g.choice([0.0, g.uniform(0, 1), 0.999]))

    def edit(x):
        x[g.random(x.shape) < share] = -np.inf
        if seed % 5 == 0:
            x[:] = np.round(x)                                 # many equal ones
    x, view = _logits(R, V, DTYPES[seed % 2], seed, spread=float(g.choice([0.1, 2, 30])), edit=edit, pad=int(g.choice([0, g.integers(1, 20)])), shift=int(g.integers(0, 9)))
    n_top = int(g.choice([0, g.integers(1, 65)]))
    tokens = g.integers(-1, V + 1, (R, int(g.integers(1, 9)))) if g.random() < 0.8 or not n_top else None
    _check(essa, ctx, x, view, tokens, n_top, float(g.choice([1.0, g.uniform(0.2, 3)])), entropy=bool(g.random() < 0.7))
