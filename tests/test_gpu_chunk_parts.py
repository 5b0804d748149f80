"""Chunk attention whose CTAs take many short parts one after the other: the accumulators, references and sums of one part give
way to the next one's while some warps are still at the end of the last.  Every column of every row is compared, over repeated
calls, which also have to be equal bit by bit.  Tolerances as in test_gpu_step.py."""
import numpy as np
import pytest
import torch

from test_gpu_step import Chunk

pytestmark = pytest.mark.gpu


def lengths(kind, n_seq, tile_tok):
    """New tokens and rows of the sequences: two row tiles each, one row tile of one to three key tiles each, or both by turns."""
    r = np.random.default_rng(tile_tok)
    two = r.integers(tile_tok + 1, 2 * tile_tok + 1, n_seq)
    one = r.integers(max(2, tile_tok - 7), tile_tok + 1, n_seq)
    new = two if kind == "two tiles" else one if kind == "one tile" else np.where(np.arange(n_seq) % 2 == 0, two, one)
    return new.tolist(), (new + r.integers(0, 330, n_seq)).tolist()


@pytest.mark.parametrize("kind", ["two tiles", "one tile", "by turns"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 1, 128), (8, 1, 64), (12, 2, 128)])
def test_many_parts_a_cta(kind, hq, hkv, d):
    new, lens = lengths(kind, 900 // hkv, 128 // (hq // hkv))
    c = Chunk(new, lens, hq, hkv, d, "bf16", seed=d + hq)
    assert sum(-(-n // (16 // (hq // hkv))) * -(-m // 128) for n, m in zip(new, lens)) * hkv > 24 * 148   # (row tiles of 128)
    first = c.call().check()
    o, lse = first.o.clone(), first.lse.clone()
    for _ in range(20):
        c.o.fill_(7)
        c.lse.fill_(7)
        c.call()
        assert torch.equal(c.o, o) and torch.equal(c.lse, lse)
