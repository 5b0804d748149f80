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


SMS = 148   # of a machine without a GPU, which is what sizes the calls here


def most_units(hq, hkv, n_seq, n_tokens, max_len):
    """bf16, from the header: items of as many tokens as fill 256 rows, one more a sequence, tiles of 128 keys and two more an item."""
    g, s = hq // hkv, min(n_seq, n_tokens)
    blocks = -(-g // 128)
    t = 2 * (128 // -(-g // blocks))
    return (n_tokens // t + s) * hkv * blocks * (-(-max_len // 128) + 2)


@pytest.mark.parametrize("hq,hkv,n_seq,n_tokens,max_len", [
    (128, 8, 64, 131072, 262144),              # 135 million units
    (32, 8, 256, 1 << 20, 262144), (8, 8, 1000, 8 << 20, 4096), (200, 1, 1, 40000, 100000), (28, 4, 65535, 65535, 131072)])
def test_bf16_capacities_within_31_bits_are_taken(lib, hq, hkv, n_seq, n_tokens, max_len):  # noqa: F811
    assert most_units(hq, hkv, n_seq, n_tokens, max_len) < 2**31
    status, size = call(lib, hq, hkv, n_seq, n_tokens, max_len)
    assert status == B.EARN_ERR_WORKSPACE
    assert size == call(lib, hq, hkv, 1, 4096, 4096)[1]          # (the parts of all SMs' shares, as for any large call)


@pytest.mark.parametrize("hq,hkv,n_seq", [(32, 8, 10), (128, 8, 1), (8, 8, 64), (200, 1, 3), (20, 4, 7)])
def test_bf16_the_last_capacity(lib, hq, hkv, n_seq):  # noqa: F811
    """The largest n_tokens that is taken, and the next one, with lists of up to 2 million rows."""
    max_len, lo, hi = 1 << 21, 1, 2**31 - 1
    while hi - lo > 1:
        mid = (lo + hi) // 2
        if most_units(hq, hkv, n_seq, mid, max_len) < 2**31:
            lo = mid
        else:
            hi = mid
    assert call(lib, hq, hkv, n_seq, lo, max_len)[0] == B.EARN_ERR_WORKSPACE
    assert call(lib, hq, hkv, n_seq, hi, max_len)[0] == B.EARN_ERR_UNSUPPORTED
    assert call(lib, hq, hkv, n_seq, 2**31 - 1, max_len)[0] == B.EARN_ERR_UNSUPPORTED
    assert call(lib, 32768, 32768, 65535, 2**31 - 1, 2**31 - 128)[0] == B.EARN_ERR_UNSUPPORTED   # (past 64 bits as well)


def test_f32_the_last_capacity(lib):  # noqa: F811
    """Row tiles of 64 rows against tiles of 64 keys: (n_tokens / 16 + 1) x 4 heads x 32768 tiles."""
    last = (2**31 // (4 * 32768) - 1) * 16 - 1
    assert call(lib, 16, 4, 1, last, 1 << 21, "f32")[0] == B.EARN_ERR_WORKSPACE
    assert call(lib, 16, 4, 1, last + 1, 1 << 21, "f32")[0] == B.EARN_ERR_UNSUPPORTED
