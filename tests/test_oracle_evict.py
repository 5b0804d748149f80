"""Pins of the evictable-cache functions of the oracle."""
import numpy as np
import pytest

from oracle import earn_oracle as orc


def _qkv(total, hq, hkv, d, seed=0):
    g = np.random.default_rng(seed)
    return g.standard_normal((total, hq, d)), g.standard_normal((total, hkv, d)), g.standard_normal((total, hkv, d))


@pytest.mark.parametrize("n_obs", [1, 3, 7, 100])
def test_key_weights_are_column_sums_of_the_causal_softmax(n_obs):
    lens, hq, hkv, d = [5, 1, 9], 4, 2, 8
    cu = np.concatenate([[0], np.cumsum(lens)])
    q, k, v = _qkv(cu[-1], hq, hkv, d)
    _, lse = orc.causal_attention(q, k, v, cu)
    w = orc.key_weights(q, k, lse, cu, n_obs)
    ref = np.zeros_like(w)
    for b, n in enumerate(lens):
        for i in range(max(0, n - n_obs), n):
            for a in range(hq):
                p = orc.attention_scores(q[cu[b] + i, a], k[cu[b]:cu[b] + i + 1, a // 2])
                ref[a // 2, cu[b]:cu[b] + i + 1] += p
        # every (row, head) pair of the window hands out a weight of one
        assert np.allclose(w[:, cu[b]:cu[b + 1]].sum(1), min(n, n_obs) * (hq // hkv))
    assert np.allclose(w, ref, rtol=1e-12, atol=1e-14)


def test_keep_rows_by_hand():
    w, pos = [0.5, 2.0, 1.0, 2.0, 0.1, 0.0], list(range(6))
    assert orc.keep_rows(w, pos, 6, 0, 0).tolist() == [0, 1, 2, 3, 4, 5]
    assert orc.keep_rows(w, pos, 2, 0, 0).tolist() == [1, 3]
    assert orc.keep_rows(w, pos, 1, 0, 0).tolist() == [1]                       # equal weights: the lower row
    assert orc.keep_rows(w, pos, 3, 1, 1).tolist() == [0, 1, 5]
    assert orc.keep_rows(w, [9, 3, 4, 5, 6, 7], 3, 4, 1).tolist() == [0, 1, 3]   # protected by position, not by row
    assert orc.keep_rows([np.nan, -np.inf, np.inf], [0, 1, 2], 2, 0, 0).tolist() == [0, 2]


def test_moves_fill_the_free_rows_in_order():
    g = np.random.default_rng(3)
    for _ in range(50):
        n, budget = int(g.integers(1, 40)), int(g.integers(1, 40))
        w, pos = g.choice([0.0, 0.25, 0.5, 1.0], n), g.permutation(n)
        keep = orc.keep_rows(w, pos, budget, 0, 0)
        src, dst = orc.evict_moves(w, pos, budget, 0, 0)
        assert len(src) == len(dst) and (np.diff(src) > 0).all() and (np.diff(dst) > 0).all()
        held = list(range(n))
        for s, t in zip(src, dst):
            held[t] = s
        assert sorted(held[:min(n, budget)]) == keep.tolist()
