"""Pins of the step oracle: hand-made tables, closed forms of the rotation, chunks against the causal prefill's oracle."""
import numpy as np

from oracle import earn_oracle as orc
from oracle import step_oracle as so


def test_tables_by_hand():
    table = np.full((4, 3), -1)
    table[0, :2] = [7, 3]
    table[1, :1] = [5]
    table[2, :3] = [1, 2, 4]
    # 20 rows grow to 33 (a third page), 5 to 16 (none), 48 are cut to 17 (one page goes back), 0 to 5 (one page)
    r = so.page_tables([33, 16, 17, 5], [20, 5, 48, 0], table, [0, 6, 9], 2, 40)
    assert r["stack"].tolist() == [0] and r["pushed"].tolist() == [0, 6, 4]
    assert r["table"][0].tolist() == [7, 3, 4] and r["table"][3, 0] == 6
    assert r["cu"].tolist() == [0, 13, 24, 24, 29] and r["seq_len"].tolist() == [33, 16, 17, 5]
    assert r["positions"][:2].tolist() == [20, 21] and r["slots"][0] == 3 * 16 + 4 and r["slots"][12] == 4 * 16
    assert r["slots"][24:29].tolist() == [96, 97, 98, 99, 100] and r["slots"][29] == -1


def test_nobody_is_overtaken():
    table = np.full((3, 4), -1)
    r = so.page_tables([33, 16, 0], [0, 0, 0], table, [0, 1], 2, 100)
    assert r["refused"] == 2 and r["seq_len"].tolist() == [0, 0, 0] and r["cu"].tolist() == [0, 33, 49, 49]
    r = so.page_tables([16, 33, 16], [0, 0, 0], table, [0, 1], 2, 100)
    assert r["refused"] == 2 and r["seq_len"].tolist() == [16, 0, 0]


def test_rotation():
    rng = np.random.default_rng(0)
    x, f = rng.standard_normal((5, 2, 8)), np.array([1.0, 0.1])
    p = np.array([0, 1, 7, 100, 3])
    for inter in (False, True):
        y = so.rotate(x, p, f, inter)
        assert np.allclose(y[0], x[0]) and np.allclose(y[:, :, 4:], x[:, :, 4:])
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
        assert np.allclose(so.rotate(y, p, f, inter, inverse=True), x)
    quarter = so.rotate(np.array([[[1.0, 0.0]]]), np.array([1]), np.array([np.pi / 2]))
    assert np.allclose(quarter, [[[0.0, 1.0]]])
    # a scalar product depends on the distance only
    a, b = x[:1], x[1:2]
    dots = [(so.rotate(a, np.array([n + 4]), f) * so.rotate(b, np.array([n]), f)).sum(-1) for n in (0, 9, 1000)]
    assert np.allclose(dots[0], dots[1]) and np.allclose(dots[0], dots[2])


def test_chunks_are_rows_of_the_prefill():
    rng = np.random.default_rng(1)
    cu = np.array([0, 9, 14], np.int32)
    q, k, v = (rng.standard_normal((14, h, 64)) for h in (4, 2, 2))
    o, lse = orc.causal_attention(q, k, v, cu)
    rows = [np.r_[5:9], np.r_[13:14]]
    got, glse, _ = so.chunk_attention(np.concatenate([q[r] for r in rows]), [k[:9], k[9:]], [v[:9], v[9:]], [4, 1], [9, 5])
    assert np.allclose(got, np.concatenate([o[r] for r in rows])) and np.allclose(glse, np.concatenate([lse[:, r] for r in rows], 1))
    none, nlse, _ = so.chunk_attention(q[:2], [k], [v], [2], [1])
    assert (none[0] == 0).all() and (nlse[:, 0] == -np.inf).all() and np.allclose(none[1, 0], v[0, 0])
