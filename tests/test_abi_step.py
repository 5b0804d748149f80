"""Host-side refusals of the calls of a step of several new tokens: nothing is launched, the binding names what it turns down."""
import ctypes as C

import pytest
import torch

from paper_2507_00715_b200 import binding as B
from test_abi_evict import MODEL, P, cache
from test_abi_host import lib  # noqa: F401  (the fixture builds the library)

ROPE = B.EarnRope(128, 0, 1.0, P)


def test_page_tables(lib):  # noqa: F811
    def call(n=2, target=P, table=P, per_seq=4, n_pages=8, held=P, free=P, n_free=P, tokens=16, cu=P, lens=P, pos=P, slots=P,
             refused=P, held_out=P, n_free_out=P, ws=P, size=512):
        pool = B.EarnPagePool(table, per_seq, n_pages, held, free, n_free)
        step = B.EarnStep(tokens, cu, lens, pos, slots, refused)
        return lib.earn_page_tables(n, target, C.byref(pool), C.byref(step), held_out, n_free_out, ws, size, None)

    n0 = lib.earn_launch_count()
    for name in ("target", "table", "held", "free", "n_free", "cu", "lens", "pos", "slots", "refused", "held_out", "n_free_out"):
        assert call(**{name: None}) == B.EARN_ERR_INVALID_ARG
        assert call(**{name: 0x1002}) == B.EARN_ERR_INVALID_ARG
    assert call(pos=0x1004) == B.EARN_ERR_INVALID_ARG
    assert call(slots=0x1008) == B.EARN_ERR_INVALID_ARG
    assert call(n=-1) == B.EARN_ERR_INVALID_ARG
    assert call(tokens=-1) == B.EARN_ERR_INVALID_ARG
    assert call(per_seq=0) == B.EARN_ERR_INVALID_ARG
    assert call(n_pages=0) == B.EARN_ERR_INVALID_ARG
    assert call(n=16385) == B.EARN_ERR_UNSUPPORTED
    assert call(per_seq=2**31 // 16) == B.EARN_ERR_UNSUPPORTED
    assert call(n_pages=2**31 // 16) == B.EARN_ERR_UNSUPPORTED
    assert call(tokens=2**31 - 1) == B.EARN_ERR_UNSUPPORTED
    assert call(ws=None) == B.EARN_ERR_WORKSPACE
    assert call(ws=0x1008) == B.EARN_ERR_WORKSPACE
    assert call(size=511) == B.EARN_ERR_WORKSPACE
    assert lib.earn_page_tables(2, P, None, None, P, P, P, 512, None) == B.EARN_ERR_INVALID_ARG
    assert call(n=0) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_rope(lib):  # noqa: F811
    def call(model=MODEL, rope=ROPE, n=3, pos=P, q=P, qs=1024, k=P, ks=256, qo=P, ko=P):
        return lib.earn_rope(C.byref(model), C.byref(rope), n, pos, q, qs, k, ks, qo, ko, 0, None)

    n0 = lib.earn_launch_count()
    for rot in (-2, 3, 130):
        assert call(rope=B.EarnRope(rot, 0, 1.0, P)) == B.EARN_ERR_INVALID_ARG
    assert call(rope=B.EarnRope(128, 0, 1.0, None)) == B.EARN_ERR_INVALID_ARG
    assert call(rope=B.EarnRope(128, 0, 1.0, 0x1004)) == B.EARN_ERR_INVALID_ARG
    assert call(rope=B.EarnRope(128, 0, -1.0, P)) == B.EARN_ERR_INVALID_ARG
    assert call(rope=B.EarnRope(128, 0, float("nan"), P)) == B.EARN_ERR_INVALID_ARG
    assert call(n=-1) == B.EARN_ERR_INVALID_ARG
    for name in ("pos", "q", "k", "qo", "ko"):
        assert call(**{name: None}) == B.EARN_ERR_INVALID_ARG
        assert call(**{name: 0x1002}) == B.EARN_ERR_INVALID_ARG
    for stride in (1023, 1028, -1024, 2**60):
        assert call(qs=stride) == B.EARN_ERR_INVALID_ARG
    assert call(ks=255) == B.EARN_ERR_INVALID_ARG
    assert call(model=B.make_model(4, 2, 8, 2, 96, "bf16")) == B.EARN_ERR_UNSUPPORTED
    assert call(n=0) == B.EARN_OK
    assert call(q=None, qo=None, k=None, ko=None) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_rope_append(lib):  # noqa: F811
    def call(model=MODEL, layer=0, rope=ROPE, n=3, pos=P, slots=P, q=P, qs=1024, k=P, ks=256, v=P, vs=256, qo=P, c=None):
        c = cache(seq_len=None) if c is None else c
        return lib.earn_rope_append(C.byref(model), layer, C.byref(rope), n, pos, slots, q, qs, k, ks, v, vs, qo, C.byref(c), None)

    n0 = lib.earn_launch_count()
    assert call(layer=2) == B.EARN_ERR_INVALID_ARG
    assert call(layer=-1) == B.EARN_ERR_INVALID_ARG
    assert call(rope=B.EarnRope(5, 0, 1.0, P)) == B.EARN_ERR_INVALID_ARG
    for name in ("pos", "slots", "q", "k", "v", "qo"):
        assert call(**{name: None}) == B.EARN_ERR_INVALID_ARG
        assert call(**{name: 0x1002}) == B.EARN_ERR_INVALID_ARG
    assert call(vs=252) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(k=None)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(n_pages=0)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(n_pages=2**31 // 16)) == B.EARN_ERR_UNSUPPORTED
    assert call(n=-1) == B.EARN_ERR_INVALID_ARG
    assert call(n=0) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_paged_chunk(lib):  # noqa: F811
    def call(model=MODEL, n=2, layer=0, tokens=10, cu=P, q=P, c=None, o=P, lse=P, ws=P, size=1 << 30):
        c = cache() if c is None else c
        return lib.earn_paged_chunk_attn(C.byref(model), n, layer, tokens, cu, q, C.byref(c), o, lse, ws, size, None)

    n0 = lib.earn_launch_count()
    assert call(layer=2) == B.EARN_ERR_INVALID_ARG
    assert call(n=-1) == B.EARN_ERR_INVALID_ARG
    assert call(tokens=-1) == B.EARN_ERR_INVALID_ARG
    assert call(n=70000, c=cache(table=P)) == B.EARN_ERR_UNSUPPORTED
    for name in ("cu", "q", "o"):
        assert call(**{name: None}) == B.EARN_ERR_INVALID_ARG
        assert call(**{name: 0x1002}) == B.EARN_ERR_INVALID_ARG
    assert call(lse=0x1002) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(seq_len=None)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(n_pages=7)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(max_len=65)) == B.EARN_ERR_INVALID_ARG
    assert call(ws=None) == B.EARN_ERR_WORKSPACE
    assert call(size=1024) == B.EARN_ERR_WORKSPACE
    assert call(model=B.make_model(4, 2, 8, 2, 96, "bf16")) == B.EARN_ERR_UNSUPPORTED
    assert call(n=0) == B.EARN_OK
    assert call(tokens=0) == B.EARN_OK
    c = cache()
    assert lib.earn_paged_chunk_workspace_bytes(C.byref(MODEL), 2, 10, C.byref(c)) > 256
    assert lib.earn_paged_chunk_workspace_bytes(C.byref(MODEL), -1, 10, C.byref(c)) == 256
    assert lib.earn_paged_chunk_workspace_bytes(C.byref(MODEL), 2, 10, C.byref(cache(max_len=0))) == 256
    assert lib.earn_launch_count() == n0


def test_the_binding_turns_down_what_the_library_cannot_see():
    x = torch.zeros(4, 6, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match=r"q: \(4, 6, 64\), expected at least \[5, 6, 64\]"):
        B._rows(x, "q", x.dtype, 5, 6, 64, -1)
    with pytest.raises(ValueError, match="one after the other"):
        B._rows(torch.zeros(6, 4, 64, dtype=x.dtype).transpose(0, 1), "q", x.dtype, 4, 6, 64, -1)
    with pytest.raises(ValueError, match="one after the other"):
        B._rows(x[:1].expand(4, 6, 64), "q", x.dtype, 4, 6, 64, -1)
    with pytest.raises(ValueError, match="k: torch.bfloat16"):
        B._rows(x, "k", torch.float32, 4, 6, 64, -1)
    assert B._rows(x[:, 2:4], "k", x.dtype, 4, 2, 64, -1) == (x[:, 2:].data_ptr(), 384)
    assert B._rows(x[:1, :2], "k", x.dtype, 1, 2, 64, -1)[1] == 128
    with pytest.raises(ValueError, match="block_table"):
        B.make_page_pool(torch.zeros(4, dtype=torch.int32), None, None, None)
