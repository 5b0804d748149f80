"""A step of several new tokens over a paged cache against the 64-bit oracle: page tables, rotary positions, chunk attention,
and a whole run of them.

Tolerances.  Rotation: the angle is reduced in 64 bits and held in 32 (2^-24 pi), sine and cosine are good to 2^-23, the
amplitude and the turn add four roundings: an element is off by at most A (|x_a| + |x_b|) 2^-21, plus one rounding to the type.
Attention: logits are sums of D products accumulated in fp32; with a = scale * max|q| * max|k| (Cauchy-Schwarz) their error is
at most (D + 4) 2^-23 a (2^-23: a matrix unit may truncate where it adds), the exponential's argument adds roundings of at most
2^-22 M with M the largest |logit|, the exponential unit 2^-22: an unnormalised weight is off by delta = (D + 4) 2^-23 a +
2^-22 max(a, M) + 2^-22, a softmax weight by 2 delta, and a sum of n terms adds n 2^-24.  With bf16 the probabilities are
rounded in front of V (2^-8 each) and the output once (2^-8).  The denominator's logarithm is off by delta + n 2^-24 and one
rounding."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2507_00715_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
PAGE = 16


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


def to64(t):
    return t.double().cpu().numpy()


def up(n):
    return -(-n // PAGE)


# ------------------------------------------------------------------------------------------------ page tables
class Pool:
    def __init__(self, held, per_seq, spare, seed=0, n_tokens=64):
        rng = np.random.default_rng(seed)
        used = sum(up(h) for h in held)
        self.n_pages = used + spare + 3
        perm = rng.permutation(self.n_pages)
        table = np.full((len(held), per_seq), -1)
        at = 0
        for b, h in enumerate(held):
            table[b, :up(h)] = perm[at:at + up(h)]
            at += up(h)
        free = np.full(self.n_pages, -1)
        free[:spare] = perm[used:used + spare]
        self.held_np, self.table_np, self.free_np, self.spare, self.n_tokens = list(held), table, free, spare, n_tokens
        self.table, self.held, self.free, self.n_free = i32(table), i32(held), i32(free), i32([spare])
        n = len(held)
        self.cu, self.seq_len, self.refused = i32(np.full(n + 1, -7)), i32(np.full(n, -7)), i32([-7])
        self.positions, self.slots = i32(np.full(n_tokens, -7)), i32(np.full(n_tokens, -7))
        self.pool = B.make_page_pool(self.table, self.held, self.free, self.n_free)
        self.step = B.make_step(self.cu, self.seq_len, self.positions, self.slots, self.refused)
        self.ws = torch.empty(B.earn_page_tables_workspace_bytes(n), dtype=torch.uint8, device="cuda")
        B.earn_workspace_init(self.ws)

    def call(self, target, in_place=True):
        held_out, n_free_out = (self.held, self.n_free) if in_place else (torch.full_like(self.held, -7), torch.full_like(self.n_free, -7))
        B.earn_page_tables(len(self.held_np), i32(target), self.pool, self.step, held_out, n_free_out, self.ws)
        return held_out, n_free_out

    def check(self, target, held_out, n_free_out):
        r = so.page_tables(target, self.held_np, self.table_np, self.free_np, self.spare, self.n_tokens)
        got = lambda t: t.cpu().numpy()  # noqa: E731
        assert (got(held_out) == r["held"]).all() and (got(self.seq_len) == r["seq_len"]).all()
        assert (got(self.cu) == r["cu"]).all() and int(self.refused) == r["refused"]
        assert (got(self.positions) == r["positions"]).all() and (got(self.slots) == r["slots"]).all()
        assert (got(self.table) == r["table"]).all()
        assert int(n_free_out) == len(r["stack"]) and (got(self.free)[:len(r["stack"])] == r["stack"]).all()
        assert (got(self.free)[len(r["pushed"]):] == self.free_np[len(r["pushed"]):]).all()   # nothing is written above the stack
        self.held_np, self.table_np, self.free_np, self.spare = list(r["held"]), r["table"], got(self.free), len(r["stack"])
        return r


@pytest.mark.parametrize("n_seq,longest,chunk,n_tokens", [(1, 40, 9, 13), (7, 100, 40, 200), (64, 300, 1, 64), (100, 200, 300, 20001),
                                                          (1024, 64, 40, 9000), (2500, 90, 3, 2600), (5000, 30, 17, 60000)])
@pytest.mark.parametrize("in_place", [True, False])
def test_page_tables(n_seq, longest, chunk, n_tokens, in_place):
    """Random steps one after the other: growth, single tokens, cuts, ends; enough pages at first, then too few."""
    rng = np.random.default_rng(n_seq + chunk)
    held = rng.integers(0, longest + 1, n_seq)
    p = Pool(held, up(longest + chunk) + 1, n_seq * up(chunk) // 2 + 1, seed=1, n_tokens=n_tokens)
    saw_refused = 0
    for _ in range(4):
        kind, h = rng.random(n_seq), np.asarray(p.held_np)
        target = np.where(kind < 0.2, h + rng.integers(1, chunk + 1, n_seq), np.where(kind < 0.7, h + 1,
                 np.where(kind < 0.9, h - rng.integers(0, 40, n_seq), 0)))
        held_out, n_free_out = p.call(target, in_place)
        r = p.check(target, held_out, n_free_out)
        saw_refused += r["refused"]
        if not in_place:
            p.held.copy_(held_out)
            p.n_free.copy_(n_free_out)
    pages = np.concatenate([p.table_np[b, :up(h)] for b, h in enumerate(p.held_np)] + [p.free_np[:p.spare]])
    assert len(set(pages.tolist())) == len(pages)                   # no page has two owners
    assert p.spare + sum(up(h) for h in p.held_np) == p.n_pages - 3


@pytest.mark.parametrize("held,target,per_seq,spare,n_tokens", [
    ([0], [1], 1, 1, 1), ([0], [0], 1, 0, 4), ([16], [17], 2, 1, 1), ([15], [16], 1, 0, 1), ([17], [16], 2, 0, 0),
    ([0, 0, 0], [33, 16, 0], 4, 2, 100),          # the first wants more than there is: nobody behind it is served
    ([0, 0], [64, 65], 4, 100, 200),              # past the table
    ([0, 0], [10, 7], 4, 100, 16), ([0, 0], [10, 6], 4, 100, 16), ([5, 5], [15, 3], 4, 9, 9),   # past the batch
    ([100, 0], [0, 100], 7, 0, 100),              # pages change hands within a call
    ([5, 5, 5], [-3, 2**31 - 1, 6], 2, 5, 8), ([], [], 1, 3, 4)])
def test_page_tables_edges(held, target, per_seq, spare, n_tokens):
    if not held:
        p = Pool([0], per_seq, spare, n_tokens=n_tokens)
        B.earn_page_tables(0, i32([0]), p.pool, p.step, p.held, p.n_free, p.ws)
        assert int(p.held) == 0 and (p.positions == -7).all()
        return
    p = Pool(held, per_seq, spare, n_tokens=n_tokens)
    p.check(target, *p.call(target))


def test_page_tables_of_a_broken_pool():
    """Counters and pages out of range: no write outside the arrays, whatever the answers are worth."""
    p = Pool([40, 0, 3], 4, 2, n_tokens=50)
    guard = torch.full((64,), 77, dtype=torch.int32, device="cuda")
    p.n_free.fill_(10 ** 6)
    p.table[0].fill_(2 ** 30)
    p.held[2] = 10 ** 6
    p.call([0, 64, 9])
    p.n_free.fill_(-5)
    p.held.fill_(-9)
    p.call([64, 64, 64])
    torch.cuda.synchronize()
    assert (guard == 77).all()


# ------------------------------------------------------------------------------------------------ rotary positions
def freqs(rot, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")


def check_turned(got, x, pos, f, interleaved, amp, inverse, dtype):
    x64 = to64(x)
    ref = so.rotate(x64, pos, f, interleaved, amp, inverse)
    rot = 2 * len(f)
    mate = np.zeros_like(x64)
    if interleaved:
        mate[..., 0:rot:2], mate[..., 1:rot:2] = x64[..., 1:rot:2], x64[..., 0:rot:2]
    else:
        mate[..., :rot // 2], mate[..., rot // 2:rot] = x64[..., rot // 2:rot], x64[..., :rot // 2]
    tol = amp * (np.abs(x64) + np.abs(mate)) * 2.0 ** -21
    tol[..., rot:] = 0
    err = np.abs(to64(got) - ref)
    assert (err <= tol + EPS[dtype] * (np.abs(ref) + tol)).all(), (err - tol).max()
    assert (to64(got)[..., rot:] == x64[..., rot:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot", [(4, 4, 64, 64), (8, 2, 128, 128), (7, 1, 128, 64), (28, 4, 128, 20), (3, 3, 64, 2),
                                          (5, 1, 64, 58), (90, 1, 128, 126), (4, 2, 128, 16), (6, 2, 64, 8)])
def test_rope(dtype, interleaved, hq, hkv, d, rot):
    """Dense rows, parts of a projection, in place; forward and gradient."""
    n, g = 37, gen(rot)
    model, f = B.make_model(1, 1, hq, hkv, d, dtype), freqs(rot)
    rope = B.make_rope(f, interleaved, 1.25)
    qkv = torch.randn(n, hq + 2 * hkv, d, generator=g, device="cuda").to(DT[dtype])
    q, k = qkv[:, :hq], qkv[:, hq:hq + hkv]
    pos = torch.randint(0, 1 << 20, (n,), generator=g, device="cuda").to(torch.int32)
    qo, ko = torch.empty(n, hq, d, device="cuda", dtype=DT[dtype]), torch.empty(n, hkv, d, device="cuda", dtype=DT[dtype])
    for inverse in (False, True):
        B.earn_rope(model, rope, n, pos, q, k, qo, ko, inverse)
        check_turned(qo, q, pos.cpu().numpy(), f.cpu().numpy(), interleaved, 1.25, inverse, dtype)
        check_turned(ko, k, pos.cpu().numpy(), f.cpu().numpy(), interleaved, 1.25, inverse, dtype)
    qc, kc = q.contiguous(), k.contiguous()
    B.earn_rope(model, rope, n, pos, qc, None, qc, None, True)
    B.earn_rope(model, rope, n, pos, None, kc, None, kc, True)
    assert torch.equal(qc, qo) and torch.equal(kc, ko)


def test_rope_far_positions_and_absent_tokens():
    n, model, f = 9, B.make_model(1, 1, 2, 1, 128, "f32"), freqs(128, 500000.0)
    rope = B.make_rope(f)
    q, k = torch.randn(n, 2, 128, device="cuda"), torch.randn(n, 1, 128, device="cuda")
    pos = i32([0, 1, 2 ** 24 + 1, 10 ** 8 + 1, 123456789, -1, 7, -2 ** 31, 3])
    qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    B.earn_rope(model, rope, n, pos, q, k, qo, ko)
    live = pos.cpu().numpy() >= 0
    check_turned(qo[live], q[live], pos.cpu().numpy()[live], f.cpu().numpy(), False, 1.0, False, "f32")
    assert (qo[~live] == 7).all() and (ko[~live] == 7).all()


def test_rope_gradient_against_differences():
    """The gradient of sum(w * rope(x)) by the call with `inverse`, against central differences of the oracle's rotation."""
    rng, f = np.random.default_rng(0), freqs(20)
    x, w, pos = rng.standard_normal((3, 2, 64)), rng.standard_normal((3, 2, 64)), np.array([5, 1000, 31])
    model = B.make_model(1, 1, 2, 2, 64, "f32")
    for inter in (False, True):
        rope, wd = B.make_rope(f, inter, 0.75), torch.tensor(w, dtype=torch.float32, device="cuda")
        dx = torch.empty_like(wd)
        B.earn_rope(model, rope, 3, i32(pos), wd, None, dx, None, inverse=True)
        for _ in range(40):
            at, h = tuple(rng.integers(0, s) for s in x.shape), 1e-3
            xp, xm = x.copy(), x.copy()
            xp[at] += h
            xm[at] -= h
            num = ((so.rotate(xp, pos, f.cpu().numpy(), inter, 0.75) - so.rotate(xm, pos, f.cpu().numpy(), inter, 0.75)) * w).sum() / (2 * h)
            assert abs(num - float(dx[at])) <= 2.0 ** -21 * 2 * np.abs(w).max() + 1e-9   # (linear in x: the difference is exact)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,rot,interleaved,n", [(8, 2, 128, 128, False, 50), (4, 4, 64, 20, False, 3), (28, 4, 128, 64, True, 300),
                                                        (6, 1, 64, 0, False, 20), (20, 4, 128, 96, False, 1)])
def test_rope_append(dtype, hq, hkv, d, rot, interleaved, n):
    g, n_pages = gen(n), up(n) + 3
    model, f = B.make_model(2, 1, hq, hkv, d, dtype), freqs(rot) if rot else None
    qkv = torch.randn(n, hq + 2 * hkv, d, generator=g, device="cuda").to(DT[dtype])
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    kp, vp = (torch.randn(n_pages, PAGE, hkv, d, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    kept_k, kept_v = kp.clone(), vp.clone()
    slots = torch.randperm(n_pages * PAGE, generator=g, device="cuda")[:n].to(torch.int32)
    pos = torch.randint(0, 4096, (n,), generator=g, device="cuda").to(torch.int32)
    out = torch.full((n, hq, d), 7.0, device="cuda", dtype=DT[dtype])
    if n > 4:
        pos[1], slots[2], slots[3] = -1, -1, n_pages * PAGE        # takes no part; dropped rows
    cache = B.make_paged_cache(kp, vp, pages_per_seq=n_pages)
    B.earn_rope_append(model, 0, B.make_rope(f, interleaved), n, pos, slots, q, k, v, out, cache)
    live = (pos >= 0).cpu().numpy()
    fn = f.cpu().numpy() if rot else np.zeros(0)
    check_turned(out[live], q[live], pos.cpu().numpy()[live], fn, interleaved, 1.0, False, dtype)
    assert (out[~live] == 7).all()
    stored = live & (slots >= 0).cpu().numpy() & (slots < n_pages * PAGE).cpu().numpy()
    at = slots.long()[stored]
    check_turned(kp.view(-1, hkv, d)[at], k[stored], pos.cpu().numpy()[stored], fn, interleaved, 1.0, False, dtype)
    assert torch.equal(vp.view(-1, hkv, d)[at], v[stored])
    rest = torch.ones(n_pages * PAGE, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert torch.equal(kp.view(-1, hkv, d)[rest], kept_k.view(-1, hkv, d)[rest])
    assert torch.equal(vp.view(-1, hkv, d)[rest], kept_v.view(-1, hkv, d)[rest])


# ------------------------------------------------------------------------------------------------ chunk attention
class Chunk:
    """Lists in shuffled pages (identity where `shuffle` is false), junk in every row that no sequence holds."""

    def __init__(self, new, lens, hq, hkv, d, dtype, seed=0, shuffle=True, scale=0.0, pad=0, junk=float("nan"), spread=1.0):
        g = gen(seed)
        dtype, _, bulk = dtype.partition(" ")
        if bulk:   # one sequence more, so long that the call goes to the kernel for many rows
            heads_a_block = -(-(hq // hkv) // -(-(hq // hkv) // 16))
            blocks, tokens, n = hkv * -(-(hq // hkv) // 16), 16 // heads_a_block, 40
            while -(-n // tokens) * up(-(-(n + 60) // 8)) * blocks <= 24 * torch.cuda.get_device_properties(0).multi_processor_count:
                n += 23
            new, lens = [*new, n], [*lens, n + 60]
        self.new, self.lens, self.hq, self.hkv, self.d, self.dtype, self.scale, self.pad = new, lens, hq, hkv, d, dtype, scale, pad
        n_seq, total = len(new), sum(new)
        self.total, per_seq = total, max(1, up(max(lens, default=0))) + 1
        self.n_pages = n_seq * per_seq + 2
        self.k, self.v = (torch.full((self.n_pages, PAGE, hkv, d), junk, device="cuda", dtype=DT[dtype]) for _ in range(2))
        order = torch.randperm(self.n_pages, generator=g, device="cuda") if shuffle else torch.arange(self.n_pages, device="cuda")
        self.table = order[:n_seq * per_seq].reshape(n_seq, per_seq).to(torch.int32)
        for b, n in enumerate(lens):
            row = torch.arange(n, device="cuda")
            at = self.table[b].long()[row // PAGE] * PAGE + row % PAGE
            self.k.view(-1, hkv, d)[at] = (spread * torch.randn(n, hkv, d, generator=g, device="cuda")).to(DT[dtype])
            self.v.view(-1, hkv, d)[at] = torch.randn(n, hkv, d, generator=g, device="cuda").to(DT[dtype])
        self.q = torch.full((total + pad, hq, d), float("nan"), device="cuda", dtype=DT[dtype])
        self.q[:total] = torch.randn(total, hq, d, generator=g, device="cuda").to(DT[dtype])
        self.cu, self.seq_len = i32(np.concatenate([[0], np.cumsum(new)])), i32(lens)
        self.o = torch.full_like(self.q, 7.0)
        self.lse = torch.full((hq, total + pad), 7.0, device="cuda")
        self.model = B.make_model(2, 1, hq, hkv, d, dtype, scale)
        self.cache = B.make_paged_cache(self.k, self.v, self.table if shuffle else None, self.seq_len, pages_per_seq=per_seq,
                                        max_len=max(1, max(lens, default=1)))
        need = B.earn_paged_chunk_workspace_bytes(self.model, n_seq, total + pad, self.cache)
        self.ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        B.earn_workspace_init(self.ws)

    def call(self, lse=True):
        B.earn_paged_chunk_attn(self.model, len(self.new), 0, self.total + self.pad, self.cu, self.q, self.cache, self.o,
                                self.lse if lse else None, self.ws)
        return self

    def rows(self, pages):
        out = []
        for b, n in enumerate(self.lens):
            row = torch.arange(n, device="cuda")
            out.append(to64(pages.view(-1, self.hkv, self.d)[self.table[b].long()[row // PAGE] * PAGE + row % PAGE]))
        return out

    def check(self, lse=True, sample=None):
        assert B.earn_device_status(self.ws) == B.EARN_OK
        k, v, q = self.rows(self.k), self.rows(self.v), to64(self.q[:self.total])
        ref, ref_lse, mag = so.chunk_attention(q, k, v, self.new, self.lens, self.scale or None)
        scale = self.scale or 1.0 / np.sqrt(self.d)
        finite = [x[np.isfinite(x).all(-1)] for x in k]
        a = scale * np.linalg.norm(q, axis=-1).max(initial=0.0) * max([np.linalg.norm(x, axis=-1).max(initial=0.0) for x in finite], default=0.0)
        n = max(self.lens, default=0)
        delta = (self.d + 4) * 2.0 ** -23 * a + 2.0 ** -22 * a + 2.0 ** -22
        bf = 2.0 ** -8 if self.dtype == "bf16" else 0.0
        tol = (2 * delta + n * 2.0 ** -24 + bf) * mag + EPS[self.dtype] * np.abs(ref)
        err = np.abs(to64(self.o[:self.total]) - ref)
        assert (err <= tol * 1.01 + 1e-30).all(), (err - tol).max()       # (1.01: the bounds' own products)
        assert (self.o[self.total:] == 7).all()
        if lse:
            got = to64(self.lse[:, :self.total])
            none = np.isneginf(ref_lse)
            assert (np.isneginf(got) == none).all()
            off = np.abs(got - ref_lse, where=~none, out=np.zeros_like(got))
            assert (off <= delta + n * 2.0 ** -24 + 2.0 ** -23 * np.abs(np.where(none, 0, ref_lse)) + 2.0 ** -23).all(), off.max()
            assert (self.lse[:, self.total:] == 7).all()
        else:
            assert (self.lse == 7).all()
        return self


HEADS = [(4, 4, 64), (8, 2, 128), (7, 1, 128), (28, 4, 64), (12, 2, 128), (3, 3, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_chunk_lengths(dtype, hq, hkv, d):
    """One token, page and tile edges, nothing new, nothing old, nothing at all, more tokens than rows, refused sequences."""
    new = [1, 0, 5, 16, 17, 1, 40, 3, 0, 9, 130, 2]
    lens = [1, 40, 5, 16, 33, 129, 168, 1, 0, 0, 131, 128]
    Chunk(new, lens, hq, hkv, d, dtype, seed=hq, pad=5).call().check()


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
@pytest.mark.parametrize("new,lens,hq,hkv,d", [
    ([1], [1], 1, 1, 64), ([1], [700], 4, 1, 128), ([5], [2005], 12, 2, 128), ([300], [300], 8, 2, 128), ([257, 255], [600, 255], 4, 4, 64),
    ([1] * 40, [(37 * i) % 300 + 1 for i in range(40)], 8, 1, 64), ([129, 1, 128], [129, 1000, 385], 2, 2, 128),
    ([70], [200], 64, 1, 64), ([33], [50], 5, 1, 128), ([64], [64], 16, 1, 128)])
def test_chunk_shapes(dtype, new, lens, hq, hkv, d):
    c = Chunk(new, lens, hq, hkv, d, dtype, seed=len(new))
    first = c.call().check().o.clone()
    c.o.fill_(7)
    assert torch.equal(c.call(lse=False).o, first)                   # equal calls, equal results


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
@pytest.mark.parametrize("hq,hkv", [(100, 1), (160, 1), (129, 1), (300, 1), (144, 2)])
def test_chunk_large_groups(dtype, hq, hkv):
    Chunk([3, 1, 0, 9], [140, 20, 5, 9], hq, hkv, 128, dtype, seed=hq).call().check()


def test_chunk_identity_table_and_scale():
    Chunk([9, 1, 50], [100, 31, 77], 8, 2, 128, "bf16", shuffle=False).call().check()
    Chunk([9, 1, 50], [100, 31, 77], 8, 2, 128, "bf16 bulk", shuffle=False, scale=0.2).call().check()
    Chunk([9, 1, 50], [100, 31, 77], 4, 2, 64, "f32", shuffle=False, scale=0.3).call().check()
    Chunk([9, 1, 50], [100, 31, 77], 4, 2, 64, "bf16", scale=0.02).call().check()


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_chunk_logits_far_apart(dtype, d):
    """Large logits, a maximum that keeps growing along the list, a first tile that lies far below the rest."""
    c = Chunk([20, 1, 3], [400, 300, 290], 8, 2, d, dtype, seed=3, spread=4.0)
    c.call().check()
    row = torch.arange(400, device="cuda")
    at = c.table[0].long()[row // PAGE] * PAGE + row % PAGE
    c.k.view(-1, 2, d)[at] *= (0.02 + row[:, None, None] / 400.0).to(c.k.dtype)
    c.call().check()


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
@pytest.mark.parametrize("new", [[300, 1, 40], [7, 1, 3]])
def test_chunk_logits_beyond_any_reference(dtype, new):
    """Keys whose logits exceed those in front of them by hundreds: late in the list, early in it, and in one list of several."""
    c = Chunk(new, [900, 300, 290], 4, 2, 128, dtype, seed=9)
    c.q[..., 0] = 4.0
    for b, far in ((0, (500, 640, 641)), (2, (40, 288))):
        row = torch.tensor(far, device="cuda")
        at = c.table[b].long()[row // PAGE] * PAGE + row % PAGE
        c.k.view(-1, 2, 128)[at, :, 0] = torch.linspace(500.0, 900.0, len(far), device="cuda").to(c.k.dtype)[:, None]
    first = c.call().check().o.clone()
    c.o.fill_(7)
    assert torch.equal(c.call().o, first)


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
def test_chunk_dead_keys(dtype):
    """Keys whose logits are -inf weigh nothing, long stretches of them at the start and whole lists included."""
    c = Chunk([6, 2, 140], [300, 40, 200], 8, 2, 128, dtype, seed=5)
    c.q[..., 0] = 0.5
    for b, n in enumerate(c.lens):
        row = torch.arange(n, device="cuda")
        dead = (row % 3 == 1) | (row < 200) if b == 0 else row >= 0 if b == 1 else (row < 64) | (row % 5 == 0)
        at = (c.table[b].long()[row // PAGE] * PAGE + row % PAGE)[dead]
        c.k.view(-1, 2, 128)[at, :, 0] = float("-inf")
    c.call().check()
    assert (c.o[6:8] == 0).all()


def test_chunk_offsets_are_cut_off():
    """Lengths and offsets out of range: no read or write outside the tensors; the rows in range are those of the cut ones."""
    c = Chunk([4, 4], [60, 60], 4, 2, 128, "bf16", pad=8)
    c.q[8:] = 0
    c.cu.copy_(i32([0, 4, 10 ** 9]))
    c.seq_len.copy_(i32([10 ** 9, -5]))
    c.call()
    assert B.earn_device_status(c.ws) == B.EARN_OK
    assert (c.o[4:] == 0).all()
    c.cu.copy_(i32([-4, 30, 2]))
    c.call()
    assert B.earn_device_status(c.ws) == B.EARN_OK


def test_chunk_offsets_of_many_rows_are_cut_off():
    c = Chunk([4], [60], 8, 2, 128, "bf16 bulk", pad=8, seed=2)
    n = c.new[1]
    c.new, c.lens = c.new[::-1], c.lens[::-1]
    c.cu.copy_(i32([0, n, n + 4]))
    c.seq_len.copy_(c.seq_len.flip(0))
    c.table.copy_(c.table.flip(0))
    c.q[n + 4:] = 0
    first = c.call().check().o.clone()
    c.cu.copy_(i32([-7, n, 10 ** 9]))
    c.call()
    assert B.earn_device_status(c.ws) == B.EARN_OK and torch.equal(c.o[:n], first[:n])
    c.cu.copy_(i32([n, 5, -1]))   # backwards: nothing is new
    c.o.fill_(7)
    c.call()
    assert B.earn_device_status(c.ws) == B.EARN_OK and (c.o == 7).all()


def test_chunk_captured_once_for_few_and_many_rows():
    """The lengths that a captured call finds on the device say which kernel does the work."""
    many = Chunk([40, 7], [200, 300], 8, 2, 128, "bf16 bulk", seed=20)
    few = [([5, 0, 30], [100, 40, 60]), ([1, 1, 1], [180, 1, 90]), ([0, 0, 0], [7, 8, 9])]
    many.call()
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            many.call()
        kept, capacity = (many.new, many.lens), many.total
        for new, lens in [few[0], kept, few[1], few[2], kept]:
            many.new, many.lens, many.total, many.pad = new, lens, sum(new), capacity - sum(new)
            many.cu.copy_(i32(np.concatenate([[0], np.cumsum(new)])))
            many.seq_len.copy_(i32(lens))
            many.o.fill_(7)
            many.lse.fill_(7)
            graph.replay()
            many.check()
    torch.cuda.current_stream().wait_stream(s)


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
def test_chunk_workspace_serves_calls_of_all_shapes(dtype):
    """One workspace for calls whose parts lie at different places, and for the block tables between them."""
    shapes = [([1] * 6, [900, 3000, 17, 2048, 1, 555]), ([300, 1], [4000, 900]), ([1], [5]), ([40, 2, 33], [1500, 16, 33]), ([1], [6000])]
    chunks = [Chunk(new, lens, 8, 2, 128, dtype, seed=i) for i, (new, lens) in enumerate(shapes)]
    ws = torch.empty(max(c.ws.numel() for c in chunks), dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(ws)
    p = Pool([3, 0], 4, 8, n_tokens=8)
    p.ws = ws
    for i in [0, 1, 2, 3, 4, 1, 0, 2, 4, 3, 0]:
        c = chunks[i]
        c.ws = ws
        c.o.fill_(7)
        c.lse.fill_(7)
        c.call().check()
        p.check([4 + i, i], *p.call([4 + i, i]))
    assert B.earn_device_status(ws) == B.EARN_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("longest", [3, 40])
def test_chunk_many_sequences(dtype, longest):
    """More sequences than a CTA keeps in shared memory."""
    r = np.random.default_rng(longest)
    new = r.integers(0, longest + 1, 1200)
    Chunk(new.tolist(), (new + r.integers(0, 30, 1200)).tolist(), 4, 2, 64, dtype, seed=8).call().check()


def test_chunk_long_chunks_and_one_long_list():
    """Items worked on by columns, and lists that every CTA has a part of."""
    Chunk([1100, 900, 1200], [1100, 1000, 1203], 28, 4, 64, "bf16", seed=9).call().check()
    Chunk([700] * 4, [700, 1300, 705, 900], 16, 16, 64, "bf16", seed=10).call().check()
    for dtype in ("bf16", "f32"):
        Chunk([1], [24001], 8, 1, 128, dtype, seed=11).call().check()
        Chunk([40], [9001], 8, 1, 128, dtype, seed=12).call().check()
    Chunk([130], [9001], 8, 1, 128, "bf16", seed=14).call().check()


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
@pytest.mark.parametrize("new,lens", [([200, 3], [900, 70]), ([1, 2], [600, 70])])
def test_chunk_rows_16_bytes_past_a_32_byte_boundary(dtype, new, lens):
    c = Chunk(new, lens, 8, 2, 64, dtype, seed=13)
    for name in ("q", "o"):
        t = getattr(c, name)
        by = 16 // t.element_size()
        moved = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")[by:].view(t.shape)
        setattr(c, name, moved.copy_(t))
    c.call().check()


@pytest.mark.parametrize("dtype", ["bf16", "bf16 bulk", "f32"])
def test_chunk_pages_behind_2_31_elements(dtype):
    """Rows stored and read behind the first 2^31 elements of the pools."""
    c = Chunk([20, 1], [60, 33], 8, 8, 128, dtype, seed=21)
    first = 2 ** 31 // (PAGE * 8 * 128) + 3
    pools = [torch.empty(first + c.n_pages, PAGE, 8, 128, device="cuda", dtype=c.k.dtype) for _ in range(2)]
    for big, small in zip(pools, (c.k, c.v)):
        big[first:] = small
    c.k, c.v = pools
    c.table += first
    c.cache = B.make_paged_cache(c.k, c.v, c.table, c.seq_len, max_len=max(c.lens))
    c.call().check()
    k, v = (torch.randn(1, 8, 128, device="cuda").to(c.k.dtype) for _ in range(2))
    slot = int(c.table[1, 0]) * PAGE + 5
    B.earn_rope_append(c.model, 0, B.make_rope(None), 1, i32([0]), i32([slot]), None, k, v, None, c.cache)
    assert torch.equal(c.k.view(-1, 8, 128)[slot], k[0]) and torch.equal(c.v.view(-1, 8, 128)[slot], v[0])


def test_chunk_two_graphs_share_a_workspace():
    """Captured calls of different shapes, replayed in turn on one stream."""
    chunks = [Chunk([3, 1, 2], [900, 3000, 40], 8, 2, 128, "bf16", seed=30), Chunk([50], [500], 8, 2, 128, "bf16 bulk", seed=31)]
    ws = torch.empty(max(c.ws.numel() for c in chunks), dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(ws)
    s, graphs = torch.cuda.Stream(), []
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for c in chunks:
            c.ws = ws
            c.call()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s):
                c.call()
        for i in (0, 1, 1, 0, 0, 1):
            chunks[i].o.fill_(7)
            chunks[i].lse.fill_(7)
            graphs[i].replay()
        for c in chunks:
            c.check()
    torch.cuda.current_stream().wait_stream(s)


def test_chunk_on_another_stream_and_captured():
    """A step captured once and replayed with other lengths, tables and offsets, on a stream of its own."""
    c = Chunk([5, 1, 40, 0], [300, 40, 90, 10], 8, 2, 128, "bf16", seed=6, pad=14)
    d = Chunk([0, 30, 1, 29], [200, 280, 1, 250], 8, 2, 128, "bf16", seed=7, pad=0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.call()
        c.o.fill_(7)
        c.lse.fill_(7)
        graph.replay()
        c.check()
        n = d.table.shape[1]
        for name in ("cu", "seq_len"):
            getattr(c, name).copy_(getattr(d, name))
        c.table[:, :n] = d.table
        c.k[:d.n_pages], c.v[:d.n_pages] = d.k, d.v
        c.q.copy_(d.q)
        c.o.fill_(7)
        c.lse.fill_(7)
        graph.replay()
        c.new, c.lens, c.total, c.pad = d.new, d.lens, d.total, 0
        c.check()
    torch.cuda.current_stream().wait_stream(s)


# ------------------------------------------------------------------------------------------------ a run of them
@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("f32", 4, 4, 64), ("bf16", 28, 4, 64)])
def test_a_run_of_steps(dtype, hq, hkv, d):
    """Prompts taken in pieces, single tokens, a rejected draft, an ended request, two layers: the outputs of the last step are
    the last rows of attention over every sequence's whole history."""
    rng, g, n_seq, room = np.random.default_rng(0), gen(1), 5, 200
    model, f = B.make_model(3, 2, hq, hkv, d, dtype), freqs(d)
    rope = B.make_rope(f)
    p = Pool([0] * n_seq, 30, 100, n_tokens=room)
    layers = [[torch.full((p.n_pages, PAGE, hkv, d), float("nan"), device="cuda", dtype=DT[dtype]) for _ in range(2)] for _ in range(2)]
    caches = [B.make_paged_cache(k, v, p.table, p.seq_len) for k, v in layers]
    ws = torch.empty(B.earn_paged_chunk_workspace_bytes(model, n_seq, room, caches[0]), dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(ws)
    history = [[[np.zeros((0, hkv, d))] * 2 for _ in range(n_seq)] for _ in range(2)]
    for step in ([100, 0, 30, 1, 7], [150, 20, 31, 2, 40], [151, 21, 60, 0, 37], [140, 22, 61, 50, 38], [145, 23, 62, 51, 39]):
        before = list(p.held_np)
        p.check(step, *p.call(step))
        for layer in range(2):
            qkv = torch.randn(room, hq + 2 * hkv, d, generator=g, device="cuda").to(DT[dtype])
            q = torch.empty(room, hq, d, device="cuda", dtype=DT[dtype])
            B.earn_rope_append(model, layer, rope, room, p.positions, p.slots, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], q, caches[layer])
            o = torch.full_like(q, 7.0)
            B.earn_paged_chunk_attn(model, n_seq, layer, room, p.cu, q, caches[layer], o, None, ws)
            assert B.earn_device_status(ws) == B.EARN_OK
            cu = p.cu.cpu().numpy()
            new = np.diff(cu)
            for b in range(n_seq):
                rows = slice(cu[b], cu[b + 1])
                kept = min(before[b], step[b])
                turned = so.rotate(to64(qkv[rows, hq:hq + hkv]), np.arange(before[b], before[b] + new[b]), f.cpu().numpy())
                h = history[layer][b]
                history[layer][b] = [np.concatenate([h[0][:kept], turned]), np.concatenate([h[1][:kept], to64(qkv[rows, hq + hkv:])])]
            q64 = np.concatenate([so.rotate(to64(qkv[cu[b]:cu[b + 1], :hq]), np.arange(before[b], before[b] + new[b]), f.cpu().numpy()) for b in range(n_seq)])
            ref, _, mag = so.chunk_attention(q64, [h[0] for h in history[layer]], [h[1] for h in history[layer]], new, step)
            err = np.abs(to64(o[:cu[-1]]) - ref)
            # two roundings of q and k to the type stand in front of the logits: |q| |k| scale 2 eps each
            a = np.linalg.norm(q64, axis=-1).max(initial=0) * max(np.linalg.norm(h[0], axis=-1).max(initial=0) for h in history[layer]) / np.sqrt(d)
            delta = (2.1 * EPS[dtype] + (d + 4) * 2.0 ** -23 + 2.0 ** -20) * a + 2.0 ** -22
            weight = np.expm1(2 * delta) + (2.0 ** -8 if dtype == "bf16" else 0) + 200 * 2.0 ** -24
            assert (err <= weight * mag + EPS[dtype] * np.abs(ref) + 1e-30).all()
            assert (o[cu[-1]:] == 7).all()
    assert p.refused.item() == 0 and rng is not None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_layers_use_the_last_page_to_its_end(dtype):
    """A greatest length inside a page: the page tables grant rows up to the page's end, and the attention has to see them."""
    from paper_2507_00715_b200.session import PagedLayers
    g = gen(3)
    q, k, v = (torch.randn(30, h, 64, generator=g, device="cuda").to(DT[dtype]) for h in (4, 2, 2))
    outs = []
    for max_len in (20, 32):
        lay = PagedLayers(1, 1, 4, 2, 64, DT[dtype], 1, 4, max_len, 30)
        lay.begin_step(i32([25]))
        outs.append(lay.layer(0, q, k, v))
        assert lay.refused() == 0 and lay.kv_entries() == 25
    assert torch.equal(outs[0], outs[1]) and not torch.equal(outs[0][24], outs[0][19])


@pytest.mark.parametrize("dtype,interleaved", [("bf16", False), ("f32", True)])
def test_paged_layers_agree_with_the_session(dtype, interleaved):
    """Prompts taken by PagedLayers in three uneven steps give the rows that a session's prefill of the whole prompts gives, and
    one more token those of its decode; then every sequence ends and the pool is full again."""
    from paper_2507_00715_b200.rope import frequencies
    from paper_2507_00715_b200.session import EarnSession, PagedLayers
    lens, hq, hkv, d, room = [200, 33, 129], 8, 2, 128, 256
    f, amp = frequencies(d, scaling="ramp", factor=2.0, original=256)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ses = EarnSession(2, 1, hq, hkv, d, DT[dtype], cu, 0, 0, max_new=1)
    lay = PagedLayers(2, 1, hq, hkv, d, DT[dtype], 3, 40, 256, room, f, interleaved, amp)
    g = gen(11)
    qkv = torch.randn(sum(lens) + 3, hq + 2 * hkv, d, generator=g, device="cuda").to(DT[dtype])   # (the last three rows: a token each)
    pos = i32(np.concatenate([np.arange(n) for n in lens] + [lens]))
    q, k = torch.empty(len(pos), hq, d, device="cuda", dtype=DT[dtype]), torch.empty(len(pos), hkv, d, device="cuda", dtype=DT[dtype])
    B.earn_rope(lay.model, lay.rope, len(pos), pos, qkv[:, :hq], qkv[:, hq:hq + hkv], q, k)
    v = qkv[:, hq + hkv:].contiguous()
    n = int(cu[-1])
    whole = ses.prefill_layer(0, q[:n], k[:n], v[:n])
    last = ses.decode_layer(0, 1, q[n:], k[n:], v[n:])
    tol = 2e-2 if dtype == "bf16" else 1e-5                # (the bounds of a single attention call on outputs of order one)
    done = [0, 0, 0]
    for target in ([70, 33, 1], [71, 33, 129], [200, 33, 129]):
        lay.begin_step(i32(target))
        rows = np.concatenate([np.arange(cu[b] + done[b], cu[b] + target[b]) for b in range(3)])
        step = torch.full((room, hq + 2 * hkv, d), float("nan"), device="cuda", dtype=DT[dtype])
        step[:len(rows)] = qkv[rows]
        o = lay.layer(0, step[:, :hq], step[:, hq:hq + hkv], step[:, hq + hkv:])
        assert lay.refused() == 0 and lay.device_status() == B.EARN_OK and lay.kv_entries() == sum(target)
        assert (o[:len(rows)].float() - whole[rows].float()).abs().max() <= 2 * tol
        assert (o[len(rows):] == 0).all()
        done = target
    lay.begin_step(i32([x + 1 for x in lens]))
    step = torch.zeros(room, hq + 2 * hkv, d, device="cuda", dtype=DT[dtype])
    step[:3] = qkv[n:]
    o = lay.layer(0, step[:, :hq], step[:, hq:hq + hkv], step[:, hq + hkv:])
    assert (o[:3].float() - last.float()).abs().max() <= 2 * tol
    lay.begin_step(i32([0, 0, 0]))
    assert int(lay.n_free) == 40 and sorted(lay.free_pages.tolist()) == list(range(40))
