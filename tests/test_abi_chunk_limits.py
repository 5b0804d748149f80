"""What a chunk attention call counts in 32 bits: the sizes from which it is refused, and those it has to take.  Nothing is
launched: a call that passes the sizes stops at its missing workspace."""
import ctypes as C

import pytest

from paper_2507_00715_b200 import binding as B
from test_abi_evict import P, cache
from test_abi_host import lib  # noqa: F401  (the fixture builds the library)


def call(lib, hq, hkv, n_seq, n_tokens, max_len, dtype="bf16", d=128):  # noqa: F811
    model = B.make_model(2, 1, hq, hkv, d, dtype)
    c = cache(table=P, per_seq=-(-max_len // 16), n_pages=8, max_len=max_len)
    n0 = lib.earn_launch_count()
    status = lib.earn_paged_chunk_attn(C.byref(model), n_seq, 0, n_tokens, P, P, C.byref(c), P, None, None, 0, None)
    assert lib.earn_launch_count() == n0
    return status, lib.earn_paged_chunk_workspace_bytes(C.byref(model), n_seq, n_tokens, C.byref(c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_a_key_tile_past_which_32_bits_end(lib, dtype):  # noqa: F811
    status, size = call(lib, 4, 1, 1, 1, 2**31 - 128, dtype)
    assert status == B.EARN_ERR_WORKSPACE and size > call(lib, 4, 1, 1, 1, 100, dtype)[1]
    for max_len in (2**31 - 112, 2**31 - 16):
        assert call(lib, 4, 1, 1, 1, max_len, dtype) == (B.EARN_ERR_UNSUPPORTED, 256)
