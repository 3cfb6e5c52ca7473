"""Masks of the oracle: a chain of drafted tokens whose words name what a causal row sees of the chain (the last `window` of it, and the sinks in it) has the causal rows' sight of
everything, however deep it is against the window."""
import numpy as np

import oracle as orc


def test_words_of_the_last_of_a_path_are_the_sliding_window():
    g = np.random.default_rng(0)
    deep = 0
    for _ in range(600):
        rows = int(g.integers(1, 20))
        L, window, sinks = rows + int(g.integers(0, 12)), int(g.integers(0, 9)), int(g.integers(0, 14))
        causal = orc.kv_mask(L, rows, window, sinks)
        assert np.array_equal(orc.kv_mask(L, rows, window, sinks, causal[:, L - rows:]), causal)
        whole = orc.kv_mask(L, rows, window, sinks, np.tril(np.ones((rows, rows), bool)))
        assert (whole >= causal)[:, L - rows:].all() and np.array_equal(whole[:, :L - rows], causal[:, :L - rows])
        deep += (whole != causal).any()
    assert deep > 100                                          # named whole, a path that is longer than the window is seen at any distance
