"""Rotary calls without tokens: nothing to do, whatever the tensors (an empty torch tensor has no address)."""
import ctypes as C

import pytest

from paper_2507_00715_b200 import binding as B
from test_abi_evict import MODEL, P, cache
from test_abi_host import lib  # noqa: F401  (the fixture builds the library)

ROPE = B.EarnRope(128, 0, 1.0, P)


@pytest.mark.parametrize("q,q_out,k,k_out", [(None, P, None, P), (P, None, P, None), (None, None, None, P), (None, None, None, None)])
def test_no_tokens(lib, q, q_out, k, k_out):  # noqa: F811
    n0 = lib.earn_launch_count()
    c = cache(seq_len=None)
    assert lib.earn_rope(C.byref(MODEL), C.byref(ROPE), 0, None, q, 0, k, 0, q_out, k_out, 0, None) == B.EARN_OK
    assert lib.earn_rope_append(C.byref(MODEL), 0, C.byref(ROPE), 0, None, None, q, 0, k, 0, None, 0, q_out, C.byref(c), None) == B.EARN_OK
    bad = B.EarnRope(3, 0, 1.0, P)
    assert lib.earn_rope(C.byref(MODEL), C.byref(bad), 0, None, q, 0, k, 0, q_out, k_out, 0, None) == B.EARN_ERR_INVALID_ARG
    assert lib.earn_launch_count() == n0
