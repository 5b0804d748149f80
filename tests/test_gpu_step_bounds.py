"""Tensors of a step between words that nobody may touch: counters, tables, offsets and lengths out of range move no write
outside the arrays, and rows in range come out as with the values cut to the range."""
import numpy as np
import pytest
import torch

from paper_2507_00715_b200 import binding as B
from test_gpu_step import Chunk, i32

pytestmark = pytest.mark.gpu
MARK, PAD = 0x5A5A5A5A, 64


class Fenced:
    """One buffer of 32-bit words; every array in it lies between PAD marked words, on a 16-byte boundary."""

    def __init__(self, **arrays):
        sizes = {name: np.asarray(a).size for name, a in arrays.items()}
        total = PAD + sum(-(-n // 4) * 4 + PAD for n in sizes.values())
        self.words = torch.full((total,), MARK, dtype=torch.int32, device="cuda")
        self.fence = torch.ones(total, dtype=torch.bool, device="cuda")
        at = PAD
        for name, a in arrays.items():
            a = np.asarray(a, dtype=np.int32)
            view = self.words[at:at + a.size]
            view.copy_(torch.as_tensor(a.reshape(-1)))
            self.fence[at:at + a.size] = False
            setattr(self, name, view.view(a.shape))
            at += -(-a.size // 4) * 4 + PAD

    def whole(self):
        return bool((self.words[self.fence] == MARK).all())


HUGE = 2 ** 31 - 1
BROKEN = {
    "more free pages than there are": dict(n_free=10 ** 6), "a negative number of free pages": dict(n_free=-5),
    "rows past the table": dict(held=[10 ** 6, 0, HUGE]), "negative rows": dict(held=[-9, -HUGE, 3]),
    "pages that do not exist": dict(table=2 ** 30), "negative pages": dict(table=-7, free=-7),
    "everything at once": dict(n_free=HUGE, held=[HUGE, -3, HUGE], table=HUGE, free=HUGE)}
TARGETS = ([0, 64, 9], [64, 64, 64], [HUGE, HUGE, HUGE], [-HUGE, 0, -1], [HUGE, 0, 64], [41, 1, 4])


@pytest.mark.parametrize("n_tokens", [50, 9000])
@pytest.mark.parametrize("what", sorted(BROKEN))
def test_page_tables(what, n_tokens):
    broken = BROKEN[what]
    n_seq, per_seq, n_pages = 3, 4, 9
    for target in TARGETS:
        table, free = np.arange(12).reshape(n_seq, per_seq) % n_pages, np.arange(n_pages)
        f = Fenced(table=np.full_like(table, broken["table"]) if "table" in broken else table,
                   free=np.full_like(free, broken["free"]) if "free" in broken else free,
                   held=broken.get("held", [40, 0, 3]), n_free=[broken.get("n_free", 2)], target=target, cu=np.zeros(n_seq + 1),
                   seq_len=np.zeros(n_seq), positions=np.zeros(n_tokens), slots=np.zeros(n_tokens), refused=[0],
                   held_out=np.zeros(n_seq), n_free_out=[0], ws=np.zeros(128))
        pool, step = B.make_page_pool(f.table, f.held, f.free, f.n_free), B.make_step(f.cu, f.seq_len, f.positions, f.slots, f.refused)
        before = f.target.clone(), f.held.clone(), f.n_free.clone()
        B.earn_page_tables(n_seq, f.target, pool, step, f.held_out, f.n_free_out, f.ws.view(torch.uint8))
        assert f.whole()
        assert all(torch.equal(x, y) for x, y in zip(before, (f.target, f.held, f.n_free)))
        assert 0 <= int(f.n_free_out) <= n_pages and 0 <= int(f.refused) <= n_seq
        cu = f.cu.tolist()
        assert cu[0] == 0 and cu == sorted(cu) and cu[-1] <= n_tokens
        assert ((f.held_out >= 0) & (f.held_out <= per_seq * 16)).all() and ((f.seq_len >= 0) & (f.seq_len <= per_seq * 16)).all()
        assert ((f.positions >= -1) & (f.positions < per_seq * 16)).all()
        assert (f.positions[cu[-1]:] == -1).all() and (f.slots[cu[-1]:] == -1).all()
        B.earn_page_tables(n_seq, f.target, pool, step, f.held, f.n_free, f.ws.view(torch.uint8))   # in place
        assert f.whole() and 0 <= int(f.n_free) <= n_pages and torch.equal(f.held, f.held_out)
        assert B.earn_device_status(f.ws.view(torch.uint8)) == B.EARN_OK


OFFSETS = [   # offsets and lengths of two sequences with room for 16 new tokens, and what they come to
    ([0, 4, 10 ** 9], [10 ** 9, -5], [0, 4, 16], [60, 0]), ([-4, 30, 2], [10 ** 9, 60], [0, 16, 16], [60, 60]),
    ([5, 3, 9], [60, 60], [3, 3, 9], [60, 60]), ([16, 5, -1], [60, 60], [0, 0, 0], [60, 60]),
    ([HUGE, HUGE, HUGE], [HUGE, HUGE], [16, 16, 16], [60, 60]), ([-HUGE, 7, 7], [33, 60], [0, 7, 7], [33, 60]),
    ([2, 2, 11], [60, 3], [2, 2, 11], [60, 3])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cu,lens,cut_cu,cut_lens", OFFSETS)
def test_chunk_offsets(dtype, cu, lens, cut_cu, cut_lens):
    c = Chunk([4, 4], [60, 60], 4, 2, 128, dtype, pad=8)
    c.q[8:] = c.q[:8].flip(0)
    rows = []
    for offsets, lengths in ((cu, lens), (cut_cu, cut_lens)):
        o = torch.full((48, 4, 128), 7.0, device="cuda", dtype=c.o.dtype)
        lse = torch.full((2 * PAD + 4 * 16,), 7.0, device="cuda")
        c.o, c.lse = o[16:32], lse[PAD:-PAD].view(4, 16)
        c.cu.copy_(i32(offsets))
        c.seq_len.copy_(i32(lengths))
        c.call()
        assert B.earn_device_status(c.ws) == B.EARN_OK
        assert (o[:16] == 7).all() and (o[32:] == 7).all() and (lse[:PAD] == 7).all() and (lse[-PAD:] == 7).all()
        rows.append((c.o.clone(), c.lse.clone()))
    assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])
    owned = torch.zeros(16, dtype=torch.bool, device="cuda")
    owned[cut_cu[0]:cut_cu[2]] = True
    assert (rows[0][0][~owned] == 7).all() and (rows[0][1][:, ~owned] == 7).all()
    assert (rows[0][0][owned] != 7).any(-1).all() and (rows[0][1][:, owned] != 7).all()


def test_chunk_offsets_of_many_rows():
    """The same for the kernel for many rows."""
    c = Chunk([], [], 8, 2, 128, "bf16 bulk", pad=24, seed=2)
    n, total = c.new[0], c.total + c.pad
    c.q[n:] = c.q[:24]
    rows = []
    for cu, lens in (([-7, 10 ** 9], [10 ** 9]), ([0, total], [n + 60]), ([9, total + 1], [n + 60]), ([9, total], [n + 60])):
        o = torch.full((total + 256, 8, 128), 7.0, device="cuda", dtype=c.o.dtype)
        lse = torch.full((2 * PAD + 8 * total,), 7.0, device="cuda")
        c.o, c.lse = o[128:-128], lse[PAD:-PAD].view(8, total)
        c.cu.copy_(i32(cu))
        c.seq_len.copy_(i32(lens))
        c.call()
        assert B.earn_device_status(c.ws) == B.EARN_OK
        assert (o[:128] == 7).all() and (o[-128:] == 7).all() and (lse[:PAD] == 7).all() and (lse[-PAD:] == 7).all()
        rows.append((c.o.clone(), c.lse.clone()))
    for a, b in ((0, 1), (2, 3)):
        assert torch.equal(rows[a][0], rows[b][0]) and torch.equal(rows[a][1], rows[b][1])
    assert (rows[2][0][:9] == 7).all() and (rows[2][1][:, :9] == 7).all() and (rows[2][0][9:] != 7).any(-1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_seq", [65535, 40000])
def test_chunk_offsets_that_give_every_token_to_thousands_of_sequences(dtype, n_seq):
    """More work than 31 bits (or 32) count, which increasing offsets cannot make: nothing is written, and the next call is right."""
    rows, heads, d = 32768, 8, 64
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.zeros(rows, heads, d, device="cuda", dtype=dt)
    o = torch.full((rows + 32, heads, d), 7.0, device="cuda", dtype=dt)
    pages = [torch.randn(8, 16, heads, d, device="cuda").to(dt) for _ in range(2)]
    table, lens = torch.zeros(n_seq, rows // 16, dtype=torch.int32, device="cuda"), torch.full((n_seq,), rows, dtype=torch.int32, device="cuda")
    cache = B.make_paged_cache(*pages, table, lens)
    cu = torch.zeros(n_seq + 1, dtype=torch.int32, device="cuda")
    cu[1::2] = rows
    model = B.make_model(2, 1, heads, heads, d, dtype)
    ws = torch.empty(B.earn_paged_chunk_workspace_bytes(model, n_seq, rows, cache), dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(ws)
    B.earn_paged_chunk_attn(model, n_seq, 0, rows, cu, q, cache, o[16:-16], None, ws)
    assert B.earn_device_status(ws) == B.EARN_OK and (o == 7).all()
    c = Chunk([40, 3], [200, 90], heads, heads, d, dtype, seed=4)
    c.ws = ws
    c.call().check()
