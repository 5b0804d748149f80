"""Host-side refusals of the evictable-cache calls: nothing is launched, and the binding names the tensor it turns down."""
import ctypes as C

import pytest
import torch

from paper_2507_00715_b200 import binding as B
from test_abi_host import FakeBatch, lib  # noqa: F401  (the fixture builds the library)

P = 0x1000


def cache(k=P, v=P, table=None, per_seq=4, n_pages=8, seq_len=P, max_len=64):
    return B.EarnPagedCache(k, v, table, per_seq, n_pages, seq_len, max_len)


MODEL = B.make_model(4, 2, 8, 2, 128, "bf16")


def test_key_weights(lib):  # noqa: F811
    ok = FakeBatch([10, 20], 2, 2)

    def call(model=MODEL, batch=ok, layer=0, n_obs=4, q=P, lse=P, w=P, ws=P, size=1 << 20):
        return lib.earn_key_weights(C.byref(model), C.byref(batch.c), layer, n_obs, q, P, lse, w, ws, size, None)

    n0 = lib.earn_launch_count()
    assert call(layer=2) == B.EARN_ERR_INVALID_ARG          # a register layer keeps its R rows
    assert call(layer=-1) == B.EARN_ERR_INVALID_ARG
    assert call(n_obs=0) == B.EARN_ERR_INVALID_ARG
    assert call(q=None) == B.EARN_ERR_INVALID_ARG
    assert call(q=0x1008) == B.EARN_ERR_INVALID_ARG
    assert call(lse=None) == B.EARN_ERR_INVALID_ARG
    assert call(w=0x1002) == B.EARN_ERR_INVALID_ARG
    assert call(ws=None) == B.EARN_ERR_WORKSPACE
    assert call(size=255) == B.EARN_ERR_WORKSPACE
    assert call(model=B.make_model(4, 2, 8, 2, 96, "bf16")) == B.EARN_ERR_UNSUPPORTED
    assert call(batch=FakeBatch([], 0, 0, max_seqlen=0)) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_evict_prompt(lib):  # noqa: F811
    ok = FakeBatch([10, 80], 2, 2)

    def call(model=MODEL, batch=ok, layer=0, policy=B.make_evict(64, 4, 4), k=P, w=P, c=None, w_out=P, pos=P, ws=P, size=1 << 30):
        c = cache() if c is None else c
        return lib.earn_evict_prompt_kv(C.byref(model), C.byref(batch.c), layer, C.byref(policy), k, P, w, C.byref(c), w_out, pos,
                                        ws, size, None)

    n0 = lib.earn_launch_count()
    assert call(layer=2) == B.EARN_ERR_INVALID_ARG
    for bad in (B.make_evict(0), B.make_evict(8, -1, 0), B.make_evict(8, 0, -1), B.make_evict(8, 5, 4),
                B.make_evict(8, 2**31 - 1, 2**31 - 1)):
        assert call(policy=bad) == B.EARN_ERR_INVALID_ARG
    assert call(policy=B.make_evict(65)) == B.EARN_ERR_INVALID_ARG        # 65 rows of the longer prompt, pages for 64
    assert call(c=cache(k=None)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(v=0x1008)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(n_pages=7)) == B.EARN_ERR_INVALID_ARG             # the identity table needs 2 x 4 pages
    assert call(c=cache(per_seq=0)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(max_len=65)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(max_len=0)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(table=0x1002)) == B.EARN_ERR_INVALID_ARG
    assert call(k=None) == B.EARN_ERR_INVALID_ARG
    assert call(w=None) == B.EARN_ERR_INVALID_ARG
    assert call(pos=None) == B.EARN_ERR_INVALID_ARG
    assert call(w_out=0x1001) == B.EARN_ERR_INVALID_ARG
    assert call(ws=None) == B.EARN_ERR_WORKSPACE
    assert call(size=256) == B.EARN_ERR_WORKSPACE
    assert call(batch=FakeBatch([], 0, 0, max_seqlen=0)) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_paged_decode(lib):  # noqa: F811
    def call(model=MODEL, n=2, layer=0, q=P, kn=P, vn=P, c=None, o=P, w=P, w_out=P, npos=P, pos=P, ws=P, size=1 << 30):
        c = cache() if c is None else c
        return lib.earn_paged_decode_attn(C.byref(model), n, layer, q, kn, vn, C.byref(c), o, w, w_out, npos, pos, ws, size, None)

    n0 = lib.earn_launch_count()
    assert call(layer=2) == B.EARN_ERR_INVALID_ARG
    assert call(n=-1) == B.EARN_ERR_INVALID_ARG
    assert call(n=70000, c=cache(table=P)) == B.EARN_ERR_UNSUPPORTED
    assert call(model=B.make_model(4, 2, 2048, 1, 128, "bf16")) == B.EARN_ERR_UNSUPPORTED   # 2048 query heads on one kv head
    assert call(q=None) == B.EARN_ERR_INVALID_ARG
    assert call(o=0x1004) == B.EARN_ERR_INVALID_ARG
    assert call(vn=None) == B.EARN_ERR_INVALID_ARG                       # a key without its value
    assert call(w_out=None) == B.EARN_ERR_INVALID_ARG                    # weights with nowhere to go
    assert call(w_out=0x1004) == B.EARN_ERR_INVALID_ARG
    assert call(npos=None) == B.EARN_ERR_INVALID_ARG
    assert call(pos=None) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(seq_len=None)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(seq_len=0x1001)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(n_pages=7)) == B.EARN_ERR_INVALID_ARG
    assert call(ws=None) == B.EARN_ERR_WORKSPACE
    assert call(size=1024) == B.EARN_ERR_WORKSPACE
    assert call(n=0) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_evict_rows(lib):  # noqa: F811
    def call(model=MODEL, n=2, layer=0, policy=B.make_evict(32, 4, 4), c=None, w=P, pos=P, w_out=P, pos_out=P, ws=P, size=1 << 30):
        c = cache() if c is None else c
        return lib.earn_evict_kv(C.byref(model), n, layer, C.byref(policy), C.byref(c), w, pos, w_out, pos_out, ws, size, None)

    n0 = lib.earn_launch_count()
    assert call(layer=2) == B.EARN_ERR_INVALID_ARG
    assert call(n=-1) == B.EARN_ERR_INVALID_ARG
    assert call(policy=B.make_evict(8, 5, 4)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(seq_len=None)) == B.EARN_ERR_INVALID_ARG
    assert call(c=cache(n_pages=0)) == B.EARN_ERR_INVALID_ARG
    for name in ("w", "pos", "w_out", "pos_out"):
        assert call(**{name: None}) == B.EARN_ERR_INVALID_ARG
        assert call(**{name: 0x1001}) == B.EARN_ERR_INVALID_ARG
    assert call(ws=0x1008) == B.EARN_ERR_WORKSPACE
    assert call(size=512) == B.EARN_ERR_WORKSPACE
    assert call(n=0) == B.EARN_OK
    assert lib.earn_launch_count() == n0


def test_workspace_size(lib):  # noqa: F811
    c = cache(per_seq=512, n_pages=1024, max_len=8192)
    need = lib.earn_paged_workspace_bytes(C.byref(MODEL), 2, C.byref(c))
    assert need >= 256 + 2 * 2 * 4 * 8192 * 4                               # one logit per (sequence, query head, row)
    assert lib.earn_paged_workspace_bytes(C.byref(MODEL), 2, C.byref(cache(max_len=0))) == 256
    assert lib.earn_paged_workspace_bytes(C.byref(MODEL), -1, C.byref(c)) == 256


def test_the_binding_turns_down_what_the_library_cannot_see():
    x = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="q: torch.bfloat16"):
        B._tensor(x, "q", torch.float32, 1, 0)
    with pytest.raises(ValueError, match="not contiguous"):
        B._tensor(x.t(), "q", torch.bfloat16, 1, 0)
    with pytest.raises(ValueError, match="at least 33"):
        B._tensor(x, "q", torch.bfloat16, 33, 0)
    with pytest.raises(ValueError, match="expected the current CUDA device"):
        B._tensor(x, "q", torch.bfloat16, 32, 0)
    with pytest.raises(ValueError, match="q: NoneType"):
        B._tensor(None, "q", torch.bfloat16, 32, 0)
    with pytest.raises(ValueError, match="n_pages"):
        B.make_paged_cache(torch.zeros(2, 8, 2, 64), torch.zeros(2, 8, 2, 64), pages_per_seq=1)
    with pytest.raises(ValueError, match="pages_per_seq"):
        B.make_paged_cache(torch.zeros(2, 16, 2, 64), torch.zeros(2, 16, 2, 64))
    other, bf16 = cache(), torch.bfloat16
    other.kind, other.n_seq, other.device = (bf16, 4, 128), 2, 0
    with pytest.raises(ValueError, match="cache of"):
        B._check_cache(MODEL, 2, other, bf16, 2, 128, 0)
    other.kind = (bf16, 2, 128)
    with pytest.raises(ValueError, match="fewer than 3"):
        B._check_cache(MODEL, 3, other, bf16, 2, 128, 0)
    with pytest.raises(ValueError, match="cache on CUDA device"):
        B._check_cache(MODEL, 2, other, bf16, 2, 128, 1)
    assert B._check_cache(MODEL, 2, other, bf16, 2, 128, 0) == 64
