"""A workspace in which another entry point has left something where the counters are: the calls say so, instead of joining
parts too early or never, and are right again after earn_workspace_init."""
import numpy as np
import pytest
import torch

from paper_2507_00715_b200 import binding as B
from test_gpu_step import Chunk, Pool

pytestmark = pytest.mark.gpu
LEFT = {"a count": 1, "two counts": 2, "a float": 0x3F000000, "a negative float": -0x41000000}


@pytest.mark.parametrize("left", sorted(LEFT))
@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
def test_chunk_attention(dtype, left):
    c = Chunk([1, 5], [6000, 900], 8, 2, 128, dtype, seed=3)
    c.call().check()
    c.ws[256:256 + 4 * 640].view(torch.int32).fill_(LEFT[left])
    c.call()
    assert B.earn_device_status(c.ws) == B.EARN_ERR_WORKSPACE
    B.earn_workspace_init(c.ws)
    assert B.earn_device_status(c.ws) == B.EARN_OK
    for _ in range(2):
        c.o.fill_(7)
        c.lse.fill_(7)
        c.call().check()


@pytest.mark.parametrize("left", sorted(LEFT))
def test_page_tables(left):
    held = [5] * 40
    p = Pool(held, 40, 1000, n_tokens=20000)      # (room for more tokens than one CTA deals with)
    target = (np.asarray(held) + 300).tolist()
    p.ws[256:].view(torch.int32).fill_(LEFT[left])
    p.call(target, in_place=False)
    assert B.earn_device_status(p.ws) == B.EARN_ERR_WORKSPACE
    q = Pool(held, 40, 1000, n_tokens=20000)
    q.ws = p.ws
    B.earn_workspace_init(q.ws)
    q.check(target, *q.call(target))
    assert B.earn_device_status(q.ws) == B.EARN_OK
