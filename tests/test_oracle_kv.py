"""The oracle of the 4-bit cache pinned by closed forms and by brute force (CPU)."""
import numpy as np

import oracle as orc


def test_format_of_simple_groups():
    x = np.zeros((1, 64), np.float32)
    x[0, :16] = np.arange(16)                                        # a range of 15: step 1, middle 8, every value exact
    q, s, m = orc.kv_quantise(x)
    assert s[0, 0] == 1 and m[0, 0] == 8 and list(q[0, :16]) == list(range(-8, 8))
    np.testing.assert_array_equal(orc.kv_values(x), x)
    np.testing.assert_array_equal(orc.kv_values(np.full((1, 64), 2.5, np.float32)), 2.5)


def test_error_is_half_a_step():
    x = np.random.default_rng(0).standard_normal((50, 2, 128)).astype(np.float32)
    q, s, m = orc.kv_quantise(x)
    err = np.abs(orc.kv_values(x) - x).reshape(50, 2, 2, 64)
    # half a step, and what rounding s (15 steps of it) and m to fp16 moves the ends of the range by
    assert (err <= s[..., None] * (0.5 + 15 * 2.0 ** -11) + np.abs(m)[..., None] * 2.0 ** -11 + 1e-6).all()
    assert q.min() == -8 and q.max() == 7


def test_groups_that_are_not_finite():
    x = np.ones((1, 128), np.float32)
    x[0, 5] = np.inf
    v = orc.kv_values(x)
    assert np.isnan(v[0, :64]).all() and (v[0, 64:] == 1).all()


def test_attention_of_equal_scores_is_the_mean():
    g = np.random.default_rng(1)
    k, v = g.standard_normal((20, 2, 64)), g.standard_normal((20, 2, 64))
    q = np.zeros((3, 4, 64))
    y, _, _ = orc.kv_attention(q, k, v, 3, 1.0)
    np.testing.assert_allclose(y[0, 1], v[:18, 0].mean(0))
    np.testing.assert_allclose(y[2, 3], v[:, 1].mean(0))
    y, _, _ = orc.kv_attention(q, k, v, 3, 1.0, window=5)
    np.testing.assert_allclose(y[1, 0], v[14:19, 0].mean(0))
    y, _, _ = orc.kv_attention(np.zeros((30, 4, 64)), k, v, 30, 1.0)
    assert (y[:10] == 0).all() and (y[10, 0] == v[0, 0]).all()


def test_pages_by_hand():
    p = orc.KvPages(5, 32, 4, 3)
    assert p.extend([1, 0], [[1] * 40, [2] * 32]) == [1, 0]
    assert p.pages[1] == [0, 1] and p.pages[0] == [2] and p.refs == [1, 1, 1, 0, 0]
    assert p.fork([1, 1], [2, 3]) == [2, 3]
    assert p.pages[2] == [0, 3] and p.pages[3] == [0, 4] and p.refs == [3, 1, 1, 1, 1]
    assert p.extend([0], [[5]]) == [orc.KV_NO_PAGES]
    assert p.fork([-1, -1], [0, 2]) == [0, 2]
    assert p.refs == [2, 1, 0, 0, 1]
    used, where = p.compact()
    assert used == 3 and where == [0, 1, -1, -1, 2] and p.pages[3] == [0, 2]
    assert p.fork([3], [3], [20]) == [3] and p.pages[3] == [3] and p.refs == [1, 1, 0, 1, 0]   # into a shared page: a copy, from the free ones


def test_a_counts_invariant():
    g = np.random.default_rng(2)
    p = orc.KvPages(60, 32, 8, 12)
    for _ in range(300):
        n = int(g.integers(1, 9))
        if g.random() < 0.5:
            p.extend([int(x) for x in g.permutation(8)[:n]], [[0] * int(k) for k in g.integers(0, 80, n)])
        else:
            p.fork([int(x) for x in g.integers(-1, 8, n)], [int(x) for x in g.permutation(8)[:n]], [int(x) for x in g.integers(-1, 200, n)])
        count = [0] * 60
        for row, tokens in zip(p.pages, p.tokens):
            assert len(row) == -(-len(tokens) // 32)
            for x in row:
                count[x] += 1
            if len(tokens) % 32:
                assert p.refs[row[-1]] == 1                          # the partly filled page is the sequence's own
        assert count == p.refs
