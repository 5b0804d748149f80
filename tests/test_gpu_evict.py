"""The evictable cache of the full layers against the fp64 oracle: key weights, the prompt's eviction into pages, decode over
the paged cache with accumulated weights, eviction in place, and a whole run of them.

Tolerances.  Logits are sums of D products accumulated in fp32; with A = scale * max|q| * max|k| (Cauchy-Schwarz) their
error is at most (D + 4) 2^-23 A (2^-23: a matrix unit may truncate where it adds), the log2-domain argument adds roundings
of at most 4 * 2^-24 * M with M the largest |logit| or |lse|, and the exponential unit 2^-22: a weight exp(logit - lse) is
off by delta = (D + 4) 2^-23 A + 2^-22 M + 2^-22 relative, a softmax weight (numerator and denominator) by 2 delta.  A sum
of n terms adds n 2^-24 relative.  With bf16 the probabilities are rounded to bf16 in front of V (2^-8 relative each) and
the output once (2^-8)."""
import numpy as np
import pytest
import torch

from oracle import earn_oracle as orc
from paper_2507_00715_b200 import binding as B
from paper_2507_00715_b200 import workloads as wl
from paper_2507_00715_b200.session import BudgetedLayers
from parity_util import assert_close, make_session, to_np

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def model_of(hq, hkv, d, dtype, scale=0.0):
    return B.make_model(2, 1, hq, hkv, d, dtype, scale)


def workspace(nbytes, fill=None):
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(ws)
    if fill is not None:
        ws[256:] = fill          # nothing behind the status block may depend on what is there
    return ws


def delta_of(qn, kn, scale, m):
    a = scale * np.linalg.norm(qn, axis=-1).max(initial=0.0) * np.linalg.norm(kn, axis=-1).max(initial=0.0)
    return (qn.shape[-1] + 4) * 2.0 ** -23 * a + 2.0 ** -22 * max(a, m) + 2.0 ** -22


# ------------------------------------------------------------------------------------------------ key weights
def run_key_weights(lens, hq, hkv, d, dtype, n_obs, seed=0, scale=0.0, garbage=False):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    g = gen(seed)
    total = int(cu[-1])
    q = torch.randn(total, hq, d, generator=g, device="cuda").to(DT[dtype])
    k = torch.randn(total, hkv, d, generator=g, device="cuda").to(DT[dtype])
    qn, kn = to_np(q), to_np(k)
    sc = scale or 1.0 / np.sqrt(d)
    _, lse64 = orc.causal_attention(qn, kn, kn, cu, scale or None)
    lse = torch.from_numpy(lse64.astype(np.float32)).cuda()
    if garbage:   # what lies outside every window is not read, or does not matter
        for b, n in enumerate(lens):
            lse[:, cu[b]:cu[b + 1] - min(n, n_obs)] = float("nan")
            q[cu[b]:cu[b + 1] - min(n, n_obs)] = float("nan")
    w = torch.full((hkv, total), 7.0, device="cuda")
    model, batch = model_of(hq, hkv, d, dtype, scale), B.Batch(cu, 0, 0)
    ws = workspace(B.earn_workspace_bytes(model, batch, 1))
    B.earn_key_weights(model, batch, 0, n_obs, q, k, lse, w, ws)
    assert B.earn_device_status(ws) == B.EARN_OK
    ref = orc.key_weights(qn, kn, lse.cpu().numpy() if not garbage else lse64.astype(np.float32), cu, n_obs, scale or None)
    tol = delta_of(qn, kn, sc, np.abs(lse64).max(initial=0.0)) + n_obs * (hq // hkv) * 2.0 ** -24 + 2.0 ** -23
    err = np.abs(w.double().cpu().numpy() - ref)
    assert (err <= tol * ref + 1e-37).all(), (err / np.maximum(ref, 1e-30)).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 2, 128), (7, 1, 128), (28, 4, 64), (20, 1, 128)])
@pytest.mark.parametrize("n_obs", [1, 5, 64, 1000])
def test_key_weights(dtype, hq, hkv, d, n_obs):
    run_key_weights([130, 1, 0, 17, 128, 300], hq, hkv, d, dtype, n_obs, seed=n_obs)


@pytest.mark.parametrize("lens,hq,hkv,n_obs", [([1], 4, 1, 1), ([3, 2], 12, 2, 2), ([600, 257, 256, 255, 513], 6, 2, 300),
                                               ([700], 1, 1, 700), ([150, 140], 100, 1, 40), ([129, 200], 160, 1, 9)])
def test_key_weights_shapes(lens, hq, hkv, n_obs):
    """A token, tile edges, one head, a group of 100 and one of 160 query heads."""
    run_key_weights(lens, hq, hkv, 128, "bf16", n_obs, seed=3)


@pytest.mark.parametrize("d", [64, 128])
def test_key_weights_ignore_what_is_outside_the_window(d):
    run_key_weights([300, 140, 5, 90], 8, 2, d, "bf16", 20, seed=4, garbage=True)
    run_key_weights([130, 40], 4, 2, d, "f32", 20, seed=4, garbage=True)


def test_key_weights_many_sequences():
    """Batches past what the block table of the short windows holds (256 sequences), and just at it; empty ones at either end."""
    run_key_weights([0, 0] + [(11 * i) % 40 for i in range(252)] + [0, 0], 4, 2, 64, "bf16", 3, seed=8)
    run_key_weights([0] + [(11 * i) % 40 for i in range(300)] + [0], 4, 2, 64, "bf16", 3, seed=9)
    run_key_weights([(131 * i) % 400 for i in range(20)], 6, 2, 128, "bf16", 400, seed=10)


@pytest.mark.parametrize("hq,d", [(48, 128), (70, 128), (43, 64)])
def test_key_weights_columns_that_no_product_fills(hq, d):
    """Groups whose tiles leave whole accumulator columns unused, after a call that left NaN in tensor memory."""
    cu = np.asarray([0, 4096], np.int32)
    q = torch.full((4096, 40, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    model, batch = model_of(40, 40, 128, "bf16"), B.Batch(cu, 0, 0)
    ws = workspace(B.earn_workspace_bytes(model, batch, 1))
    B.earn_prefill_attn(model, batch, 0, q, q, q, torch.empty_like(q), None, ws)
    run_key_weights([300, 140], hq, 1, d, "bf16", 12, seed=hq)


@pytest.mark.parametrize("hq,hkv,d,n_obs", [(8, 2, 128, 400), (7, 1, 128, 400), (7, 1, 64, 20), (48, 1, 128, 30), (100, 1, 128, 9)])
def test_key_weights_of_keys_that_overflow(hq, hkv, d, n_obs):
    """Keys whose logit is -inf under every query have a weight of 0, whatever columns the group leaves unused; a -inf logit is
    one of the inputs' own (an infinite channel against a positive query), so the others' tolerance is that of finite keys."""
    lens = [300, 140]
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    g = gen(hq)
    q = torch.randn(int(cu[-1]), hq, d, generator=g, device="cuda").to(torch.bfloat16)
    k = torch.randn(int(cu[-1]), hkv, d, generator=g, device="cuda").to(torch.bfloat16)
    q[..., 0] = 0.5
    finite = to_np(k)
    dead = torch.arange(int(cu[-1]), device="cuda") % 3 == 1
    dead[:cu[1] - 100] |= torch.arange(int(cu[1]) - 100, device="cuda") >= 64    # a long stretch of them, too
    k[dead, :, 0] = float("-inf")
    qn, kn = to_np(q), to_np(k)
    _, lse64 = orc.causal_attention(qn, kn, np.zeros_like(kn), cu)
    lse = torch.from_numpy(lse64.astype(np.float32)).cuda()
    w = torch.full((hkv, int(cu[-1])), 7.0, device="cuda")
    model, batch = model_of(hq, hkv, d, "bf16"), B.Batch(cu, 0, 0)
    ws = workspace(B.earn_workspace_bytes(model, batch, 1))
    B.earn_key_weights(model, batch, 0, n_obs, q, k, lse, w, ws)
    ref = orc.key_weights(qn, kn, lse.cpu().numpy(), cu, n_obs)
    tol = delta_of(qn, finite, 1.0 / np.sqrt(d), np.abs(lse64).max()) + n_obs * (hq // hkv) * 2.0 ** -24 + 2.0 ** -23
    got = w.double().cpu().numpy()
    assert (got[:, dead.cpu().numpy()] == 0).all()
    assert (np.abs(got - ref) <= tol * ref + 1e-37).all()


def test_key_weights_other_scale():
    run_key_weights([200, 131], 4, 2, 128, "bf16", 50, seed=5, scale=0.25)


# ------------------------------------------------------------------------------------------------ the paged pool
class Pool:
    """A page pool with a scattered table; rows of sequence b as [cap, Hkv, D] through rows(b)."""

    def __init__(self, n_seq, hkv, d, dtype, per_seq, seed=0, identity=False, spare=3):
        g = gen(1000 + seed)
        self.n_seq, self.hkv, self.d, self.per_seq, self.cap = n_seq, hkv, d, per_seq, 16 * per_seq
        n_pages = n_seq * per_seq + spare
        self.k = torch.randn(n_pages, 16, hkv, d, generator=g, device="cuda").to(DT[dtype])
        self.v = torch.randn(n_pages, 16, hkv, d, generator=g, device="cuda").to(DT[dtype])
        self.table = None if identity else torch.randperm(n_pages, generator=g, device="cuda")[:n_seq * per_seq].to(torch.int32).reshape(n_seq, per_seq)

    def cache(self, lens, max_len=None):
        self.seq_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        return B.make_paged_cache(self.k, self.v, self.table, self.seq_len, max_len, self.per_seq)

    def pages(self, b):
        return torch.arange(b * self.per_seq, (b + 1) * self.per_seq, device="cuda") if self.table is None else self.table[b].long()

    def rows(self, pool, b):
        return pool[self.pages(b)].reshape(self.cap, self.hkv, self.d)


# ------------------------------------------------------------------------------------------------ decode
def run_decode(lens, hq, hkv, d, dtype, weigh=True, in_place=False, fresh=True, start=True, identity=False, max_len=None, seed=0,
               spread=1.0, extra_pages=1, positions=True):
    n_seq = len(lens)
    pool = Pool(n_seq, hkv, d, dtype, -(-max(max(lens), 1) // 16) + extra_pages, seed, identity)
    cache = pool.cache(lens, max_len)
    g = gen(seed)
    q = (spread * torch.randn(n_seq, hq, d, generator=g, device="cuda")).to(DT[dtype])
    kn = torch.randn(n_seq, hkv, d, generator=g, device="cuda").to(DT[dtype])
    vn = torch.randn(n_seq, hkv, d, generator=g, device="cuda").to(DT[dtype])
    o = torch.full_like(q, 9.0)
    w0 = torch.rand(n_seq, hkv, pool.cap, generator=g, device="cuda") if weigh and start else None
    w1 = None if not weigh else w0 if in_place else torch.full((n_seq, hkv, pool.cap), -3.0, device="cuda")
    before = None if w0 is None else w0.clone()
    pos = torch.full((n_seq, hkv, pool.cap), -5, dtype=torch.int32, device="cuda") if positions else None
    new_pos = torch.arange(100, 100 + n_seq, dtype=torch.int32, device="cuda") if positions else None
    k0, v0 = pool.k.clone(), pool.v.clone()
    model = model_of(hq, hkv, d, dtype)
    ws = workspace(B.earn_paged_workspace_bytes(model, n_seq, cache), fill=0xff)
    B.earn_paged_decode_attn(model, n_seq, 0, q, kn if fresh else None, vn if fresh else None, cache, o, w0, w1, new_pos, pos, ws)
    assert B.earn_device_status(ws) == B.EARN_OK
    qn, sc = to_np(q), 1.0 / np.sqrt(d)
    for b, n in enumerate(lens):
        if fresh and n > 0:                                  # the appended row, and nothing else, has changed
            at = pool.pages(b)[(n - 1) // 16]
            k0[at, (n - 1) % 16], v0[at, (n - 1) % 16] = kn[b], vn[b]
        ks, vs = to_np(pool.rows(k0, b)[:n]), to_np(pool.rows(v0, b)[:n])
        ref, step = orc.paged_decode(qn[b], ks, vs)
        dl = 2 * delta_of(qn[b], ks, sc, 0.0) + n * 2.0 ** -23
        grp = hq // hkv
        av = np.zeros_like(ref)
        for a in range(hq if n else 0):
            av[a] = orc.attention_scores(qn[b, a], ks[:, a // grp]) @ np.abs(vs[:, a // grp])
        tol = (dl + (2.0 ** -8 if dtype == "bf16" else 0.0)) * av + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -23) * np.abs(ref) + 1e-37
        err = np.abs(o[b].double().cpu().numpy() - ref)
        assert (err <= tol).all(), (b, n, (err - tol).max())
        if weigh:
            got = w1[b].double().cpu().numpy()
            base = np.zeros((hkv, n)) if not start else before[b, :, :n].double().cpu().numpy()
            if fresh and n > 0:
                base[:, n - 1] = 0.0
            err = np.abs(got[:, :n] - (base + step))
            assert (err <= dl * step + 2.0 ** -23 * (base + step) + 1e-37).all(), (b, n)
            rest = before[b, :, n:] if in_place else torch.full_like(w1[b, :, n:], -3.0)
            assert torch.equal(w1[b, :, n:], rest)
        if positions:
            want = torch.full((hkv, pool.cap), -5, dtype=torch.int32, device="cuda")
            if n > 0:
                want[:, n - 1] = 100 + b
            assert torch.equal(pos[b], want)
    assert torch.equal(pool.k, k0) and torch.equal(pool.v, v0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 2, 128), (7, 1, 128), (28, 4, 64), (40, 2, 128), (17, 1, 64)])
def test_decode(dtype, hq, hkv, d):
    run_decode([0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 100], hq, hkv, d, dtype)
    run_decode([700, 5, 0, 1025], hq, hkv, d, dtype, in_place=True, seed=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(weigh=False), dict(fresh=False), dict(start=False), dict(identity=True), dict(positions=False),
                                dict(extra_pages=0), dict(weigh=False, fresh=False, positions=False), dict(spread=8.0)])
def test_decode_variants(dtype, kw):
    run_decode([1, 16, 257, 0, 530], 8, 2, 128, dtype, seed=2, **kw)
    run_decode([3], 6, 2, 64, dtype, seed=3, **kw)


@pytest.mark.parametrize("lens", [[1], [512], [2048], [2049], [6000, 1, 5999], [33000]])
def test_decode_lengths(lens):
    run_decode(lens, 8, 2, 128, "bf16", seed=4)


def test_decode_many_sequences():
    run_decode([(37 * i) % 300 for i in range(300)], 4, 1, 128, "bf16", seed=5)
    run_decode([(7 * i) % 20 for i in range(2500)], 1, 1, 64, "bf16", seed=6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_many_heads(dtype):
    run_decode([40, 3, 0], 1024, 1, 64, dtype, seed=7)        # the largest group
    run_decode([33, 700], 128, 64, 64, dtype, seed=8)


def test_decode_length_past_the_bound_counts_as_the_bound():
    """seq_len above max_len: the list ends at max_len, nothing past it is touched."""
    hq, hkv, d = 4, 2, 128
    pool = Pool(2, hkv, d, "bf16", 4)
    q = torch.randn(2, hq, d, generator=gen(1), device="cuda").to(torch.bfloat16)
    model, o, o2 = model_of(hq, hkv, d, "bf16"), torch.empty_like(q), torch.empty_like(q)
    for lens, out in (([1000, -7], o), ([40, 0], o2)):
        cache = pool.cache(lens, 40)
        ws = workspace(B.earn_paged_workspace_bytes(model, 2, cache))
        B.earn_paged_decode_attn(model, 2, 0, q, None, None, cache, out, workspace=ws)
    assert torch.equal(o, o2) and o[1].abs().sum() == 0


def test_decode_with_a_corrupt_table_stays_inside_the_pool():
    """Page numbers outside the pool: reads are clamped, the append is dropped; the other sequences do not notice."""
    hq, hkv, d = 4, 2, 128
    for dtype in ("bf16", "f32"):
        pool = Pool(3, hkv, d, dtype, 3)
        lens = [40, 33, 48]
        q, kn, vn = (torch.randn(3, h, d, generator=gen(i), device="cuda").to(DT[dtype]) for i, h in ((1, hq), (2, hkv), (3, hkv)))
        model, outs, pools = model_of(hq, hkv, d, dtype), [], []
        for bad in (False, True):
            p = Pool(3, hkv, d, dtype, 3)
            if bad:
                p.table[1] = torch.tensor([-1, 2 ** 30, -2 ** 31], dtype=torch.int32)
            cache = p.cache(lens)
            ws = workspace(B.earn_paged_workspace_bytes(model, 3, cache))
            o = torch.empty_like(q)
            B.earn_paged_decode_attn(model, 3, 0, q, kn, vn, cache, o, workspace=ws)
            torch.cuda.synchronize()
            outs.append(o)
            pools.append(p)
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][2], outs[1][2])
        changed = (pools[1].k != pool.k).flatten(1).any(1).nonzero().flatten().tolist()
        assert sorted(changed) == sorted([int(pool.table[0, 2]), int(pool.table[2, 2])])


def test_decode_masked_places_may_hold_anything():
    """NaN and infinity in the pages behind the list, and -inf logits: neither reaches a result."""
    hq, hkv, d = 8, 2, 128
    for dtype in ("bf16", "f32"):
        pool = Pool(2, hkv, d, dtype, 3)
        lens = [19, 33]
        model = model_of(hq, hkv, d, dtype)
        q = torch.randn(2, hq, d, generator=gen(1), device="cuda").to(DT[dtype])
        outs = []
        for junk in (0.0, float("nan"), float("inf")):
            for b, n in enumerate(lens):
                for pg in range(3):
                    for s in range(16):
                        if pg * 16 + s >= n:
                            pool.k[pool.table[b, pg].long(), s] = junk
                            pool.v[pool.table[b, pg].long(), s] = junk
            cache = pool.cache(lens)
            ws = workspace(B.earn_paged_workspace_bytes(model, 2, cache), fill=0xff)
            o, w = torch.empty_like(q), torch.zeros(2, hkv, pool.cap, device="cuda")
            B.earn_paged_decode_attn(model, 2, 0, q, None, None, cache, o, None, w, None, None, ws)
            outs.append((o, w))
        for o, w in outs[1:]:
            assert torch.equal(o, outs[0][0]) and torch.equal(w, outs[0][1])


@pytest.mark.parametrize("n", [100, 1500, 5000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_of_keys_that_overflow(dtype, n):
    """Whole tiles of rows with a logit of -inf, the first ones among them, get no weight and change no output."""
    hq, hkv, d = 8, 2, 128
    pool = Pool(1, hkv, d, dtype, -(-n // 16), seed=3)
    cache = pool.cache([n])
    g = gen(3)
    q = torch.randn(1, hq, d, generator=g, device="cuda").to(DT[dtype])
    q[..., 0] = 0.5
    live = pool.rows(pool.k, 0).clone()
    dead = torch.zeros(pool.cap, dtype=torch.bool, device="cuda")
    dead[:n // 3] = True
    dead[n // 2::2] = True
    k = live.clone()
    k[dead, :, 0] = float("-inf")
    pool.k[pool.pages(0)] = k.reshape(-1, 16, hkv, d)
    o = torch.empty_like(q)
    w = torch.empty(1, hkv, pool.cap, device="cuda")
    model = model_of(hq, hkv, d, dtype)
    ws = workspace(B.earn_paged_workspace_bytes(model, 1, cache), fill=0xff)
    B.earn_paged_decode_attn(model, 1, 0, q, None, None, cache, o, None, w, None, None, ws)
    qn, ks, vs, gone = to_np(q[0]), to_np(live[:n]), to_np(pool.rows(pool.v, 0)[:n]), dead[:n].cpu().numpy()
    ref, step = orc.paged_decode(qn, ks[~gone], vs[~gone])
    dl = 2 * delta_of(qn, ks, 1.0 / np.sqrt(d), 0.0) + n * 2.0 ** -23
    rnd = 2.0 ** -8 if dtype == "bf16" else 0.0
    av = np.stack([orc.attention_scores(qn[a], ks[~gone][:, a // 4]) @ np.abs(vs[~gone][:, a // 4]) for a in range(hq)])
    got, wn = o[0].double().cpu().numpy(), w[0, :, :n].double().cpu().numpy()
    assert (np.abs(got - ref) <= (dl + rnd) * av + max(rnd, 2.0 ** -23) * np.abs(ref) + 1e-37).all()
    assert (wn[:, gone] == 0).all()
    assert (np.abs(wn[:, ~gone] - step) <= (dl + 4 * 2.0 ** -24) * step + 1e-37).all()


def test_decode_offsets_past_32_bits():
    """A pool of more than 2^31 elements (4.3 GB a tensor), the sequence's pages at its end."""
    hq, hkv, d = 8, 8, 128
    n_pages = 2 ** 31 // (16 * hkv * d) + 8
    k = torch.zeros(n_pages, 16, hkv, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    tail = torch.arange(n_pages - 4, n_pages, dtype=torch.int32, device="cuda").reshape(1, 4)
    k[-4:] = torch.randn(4, 16, hkv, d, generator=gen(1), device="cuda").to(torch.bfloat16)
    v[-4:] = torch.randn(4, 16, hkv, d, generator=gen(2), device="cuda").to(torch.bfloat16)
    q = torch.randn(1, hq, d, generator=gen(3), device="cuda").to(torch.bfloat16)
    kn, vn = q.clone(), -q
    seq_len = torch.tensor([60], dtype=torch.int32, device="cuda")
    model = model_of(hq, hkv, d, "bf16")
    small_k, small_v = k[-4:].clone(), v[-4:].clone()
    outs = []
    for kp, vp, table in ((k, v, tail), (small_k, small_v, tail - (n_pages - 4))):
        cache = B.make_paged_cache(kp, vp, table, seq_len)
        ws = workspace(B.earn_paged_workspace_bytes(model, 1, cache))
        o, w = torch.empty_like(q), torch.rand(1, hkv, 64, generator=gen(5), device="cuda")
        pos = torch.arange(64, dtype=torch.int32, device="cuda").expand(1, hkv, 64).contiguous()
        B.earn_paged_decode_attn(model, 1, 0, q, kn, vn, cache, o, w, w, torch.tensor([59], dtype=torch.int32, device="cuda"), pos, ws)
        B.earn_evict_kv(model, 1, 0, B.make_evict(20, 2, 2), cache, w, pos, w, pos, ws)
        outs.append((o, w, pos, kp[-4:], vp[-4:]))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert k[:-4].abs().amax() == 0


# ------------------------------------------------------------------------------------------------ eviction, prompt form
def weights_of(shape, g, kind):
    w = torch.exp(2.0 * torch.randn(shape, generator=g, device="cuda"))
    if kind == "ties":
        w = (w * 2).round().clamp(max=3.0) * 0.5
    elif kind == "zeros":
        w = torch.zeros_like(w)
    elif kind == "odd":
        pick = torch.randint(0, 12, shape, generator=g, device="cuda")
        for i, x in enumerate((float("nan"), float("inf"), float("-inf"), -0.0, 0.0, -1.5, 1e-42, -1e-42)):
            w[pick == i] = x
    return w


@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 2, 128), ("f32", 3, 64), ("bf16", 1, 64), ("f32", 2, 128)])
@pytest.mark.parametrize("kind", ["tail", "ties", "zeros", "odd"])
@pytest.mark.parametrize("budget,n_first,n_last", [(1, 0, 0), (1, 1, 0), (20, 4, 4), (64, 64, 0), (64, 0, 64), (100, 3, 30)])
def test_evict_prompt(dtype, hkv, d, kind, budget, n_first, n_last):
    lens = [0, 1, 19, 20, 21, 64, 65, 300, 2500]
    run_evict_prompt(lens, dtype, hkv, d, kind, budget, n_first, n_last)


def run_evict_prompt(lens, dtype, hkv, d, kind, budget, n_first, n_last, identity=False, carry=True):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    g, total, n_seq = gen(budget), int(cu[-1]), len(lens)
    k = torch.randn(total, hkv, d, generator=g, device="cuda").to(DT[dtype])
    v = torch.randn(total, hkv, d, generator=g, device="cuda").to(DT[dtype])
    w = weights_of((hkv, total), g, kind)
    pool = Pool(n_seq, hkv, d, dtype, -(-min(max(lens), budget) // 16) + 1, identity=identity)
    k0, v0 = pool.k.clone(), pool.v.clone()
    cache = pool.cache([0] * n_seq)
    w_out = torch.full((n_seq, hkv, pool.cap), -3.0, device="cuda") if carry else None
    pos = torch.full((n_seq, hkv, pool.cap), -5, dtype=torch.int32, device="cuda")
    model, batch = model_of(hkv, hkv, d, dtype), B.Batch(cu, 0, 0)
    ws = workspace(B.earn_paged_workspace_bytes(model, n_seq, cache), fill=0xff)
    B.earn_evict_prompt_kv(model, batch, 0, B.make_evict(budget, n_first, n_last), k, v, w, cache, w_out, pos, ws)
    assert B.earn_device_status(ws) == B.EARN_OK
    wn = w.cpu().numpy()
    for b, n in enumerate(lens):
        for h in range(hkv):
            keep = torch.from_numpy(orc.keep_rows(wn[h, cu[b]:cu[b + 1]], np.arange(n), budget, n_first, n_last)).cuda() if n else torch.zeros(0, dtype=torch.int64, device="cuda")
            m = keep.numel()
            assert torch.equal(pos[b, h, :m].long(), keep) and (pos[b, h, m:] == -5).all(), (b, h)
            if carry:
                assert torch.equal(w_out[b, h, :m].view(torch.int32), w[h, cu[b] + keep].view(torch.int32)) and (w_out[b, h, m:] == -3.0).all()
            page, slot = pool.pages(b)[torch.arange(m, device="cuda") // 16], torch.arange(m, device="cuda") % 16
            k0[page, slot, h], v0[page, slot, h] = k[cu[b] + keep, h], v[cu[b] + keep, h]
    assert torch.equal(pool.k, k0) and torch.equal(pool.v, v0)


def test_evict_prompt_variants():
    run_evict_prompt([100, 40], "bf16", 2, 128, "tail", 32, 2, 2, identity=True, carry=False)
    run_evict_prompt([60000, 50], "bf16", 1, 64, "ties", 9000, 16, 64)
    run_evict_prompt([60000], "bf16", 1, 64, "zeros", 30000, 0, 5)
    run_evict_prompt([70000, 7], "bf16", 1, 64, "ties", 5000, 16, 64)        # a list past what a cluster holds
    run_evict_prompt([66000], "bf16", 1, 64, "odd", 300, 16, 64)
    run_evict_prompt([65536, 65535, 7], "bf16", 1, 64, "tail", 5000, 16, 64)
    run_evict_prompt([32768, 32767, 5], "bf16", 1, 64, "ties", 3000, 16, 64)
    run_evict_prompt([9000, 2000, 100], "f32", 2, 128, "ties", 50, 0, 0)
    run_evict_prompt([21, 40, 19, 20, 28, 0, 300] * 86 + [33], "bf16", 1, 64, "ties", 20, 2, 2)   # more than are resident at once
    run_evict_prompt([10, 3], "bf16", 2, 128, "tail", 2 ** 31 - 1, 2, 2)     # a budget nothing reaches


# ------------------------------------------------------------------------------------------------ eviction in place
def run_evict(lens, dtype, hkv, d, kind, budget, n_first, n_last, in_place=True, identity=False, max_len=None, seed=0):
    n_seq = len(lens)
    pool = Pool(n_seq, hkv, d, dtype, -(-max(lens) // 16) + 1, seed, identity)
    cache = pool.cache(lens, max_len)
    g = gen(seed)
    w = weights_of((n_seq, hkv, pool.cap), g, kind)
    pos = torch.stack([torch.randperm(pool.cap, generator=g, device="cuda") for _ in range(n_seq * hkv)]).to(torch.int32).reshape(n_seq, hkv, pool.cap)
    w_in, p_in = w.clone(), pos.clone()
    w_out = w if in_place else torch.full_like(w, -3.0)
    p_out = pos if in_place else torch.full_like(pos, -5)
    want_w, want_p = w_out.clone(), p_out.clone()
    k0, v0 = pool.k.clone(), pool.v.clone()
    model = model_of(hkv, hkv, d, dtype)
    ws = workspace(B.earn_paged_workspace_bytes(model, n_seq, cache), fill=0xff)
    B.earn_evict_kv(model, n_seq, 0, B.make_evict(budget, n_first, n_last), cache, w, pos, w_out, p_out, ws)
    assert B.earn_device_status(ws) == B.EARN_OK
    wn, pn = w_in.cpu().numpy(), p_in.cpu().numpy()
    for b, n in enumerate(lens):
        left = min(n, budget)
        for h in range(hkv):
            want_w[b, h, :left], want_p[b, h, :left] = w_in[b, h, :left], p_in[b, h, :left]
            if n <= budget:
                continue
            src, dst = (torch.from_numpy(x).cuda() for x in orc.evict_moves(wn[b, h, :n], pn[b, h, :n], budget, n_first, n_last))
            want_w[b, h, dst], want_p[b, h, dst] = w_in[b, h, src], p_in[b, h, src]
            pg = pool.pages(b)
            k0[pg[dst // 16], dst % 16, h], v0[pg[dst // 16], dst % 16, h] = k0[pg[src // 16], src % 16, h], v0[pg[src // 16], src % 16, h]
    assert torch.equal(p_out, want_p)
    assert torch.equal(w_out.view(torch.int32), want_w.view(torch.int32))
    assert torch.equal(pool.k, k0) and torch.equal(pool.v, v0)


@pytest.mark.parametrize("dtype,hkv,d", [("bf16", 2, 128), ("f32", 3, 64), ("bf16", 1, 64), ("f32", 2, 128)])
@pytest.mark.parametrize("kind", ["tail", "ties", "zeros", "odd"])
@pytest.mark.parametrize("budget,n_first,n_last", [(1, 0, 0), (20, 4, 4), (64, 0, 64), (300, 30, 30)])
def test_evict(dtype, hkv, d, kind, budget, n_first, n_last):
    run_evict([0, 1, 19, 20, 21, 65, 301, 2500], dtype, hkv, d, kind, budget, n_first, n_last)
    run_evict([21, 3, 400, 64], dtype, hkv, d, kind, budget, n_first, n_last, in_place=False, seed=1)


def test_evict_variants():
    run_evict([33, 64, 50], "bf16", 2, 128, "tail", 32, 4, 4, identity=True)
    run_evict([60000, 9], "bf16", 1, 64, "ties", 20000, 16, 64)
    run_evict([70000, 9, 66000], "bf16", 1, 64, "ties", 20000, 16, 64)       # a list past what a cluster holds
    run_evict([70000, 9], "bf16", 1, 64, "odd", 40000, 16, 64, in_place=False)
    run_evict([65536], "bf16", 1, 64, "tail", 65535, 16, 64)
    run_evict([60000, 9], "bf16", 1, 64, "tail", 20000, 16, 64, in_place=False)
    run_evict([40000, 9], "bf16", 1, 64, "odd", 20000, 16, 64)
    run_evict([32768, 9, 20000], "bf16", 1, 64, "ties", 9000, 16, 64)
    run_evict([9000, 4100, 100], "f32", 2, 128, "zeros", 4096, 3, 40, in_place=False)
    # more lists than are resident at once, long and hardly too long ones among them: the moves go to a second kernel
    run_evict([21, 40, 19, 20, 28, 29, 300] * 86 + [33], "bf16", 1, 64, "ties", 20, 2, 2)
    run_evict([21, 40, 19, 20, 28, 29, 300] * 86 + [33], "f32", 1, 64, "tail", 20, 2, 2, in_place=False)
    for excess in range(1, 10):                                              # few rows too many, some or all behind the budget
        run_evict([300 + excess, 299, 301], "bf16", 2, 64, "odd", 300, 0, 0, in_place=excess % 2 == 0, seed=excess)
        run_evict([40 + excess, 39, 41], "f32", 1, 64, "zeros", 40, 20, 20, seed=excess)
    run_evict([100, 20], "bf16", 2, 128, "tail", 2 ** 31 - 1, 4, 4)          # a budget nothing reaches
    run_evict([1025] * 7, "bf16", 3, 128, "tail", 1024, 16, 64)              # a step's worth


# ------------------------------------------------------------------------------------------------ the whole run
def _reference_step(state, q, kn, vn, pos):
    """Oracle state per (sequence, head): keys, values, weight, position lists; one decode step."""
    outs = []
    for b, heads in enumerate(state):
        grp = q.shape[1] // len(heads)
        o = np.zeros(q.shape[1:])
        for h, st in enumerate(heads):
            st["k"].append(kn[b, h])
            st["v"].append(vn[b, h])
            st["w"].append(0.0)
            st["pos"].append(pos[b])
            oo, w = orc.paged_decode(q[b, h * grp:(h + 1) * grp], np.asarray(st["k"])[:, None], np.asarray(st["v"])[:, None])
            o[h * grp:(h + 1) * grp] = oo
            st["w"] = [float(x) for x in np.asarray(st["w"]) + w[0]]
        outs.append(o)
    return np.stack(outs)


@pytest.mark.parametrize("graph", [False, True])
def test_prompt_then_steps_at_the_budget(graph):
    """Prefill with lse -> key weights -> eviction into pages -> steps of decode and eviction, as a serving loop runs them
    (in place, one workspace, seq_len on the device), eagerly and with the step captured once and replayed.  The choice of
    rows is checked against the oracle on the weights that the library computed; the values against the oracle's cache."""
    lens, hq, hkv, d, budget, n_first, n_last, steps = [150, 40, 97], 8, 2, 128, 48, 4, 6, 5
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total, n_seq, g = int(cu[-1]), len(lens), gen(11)
    q, k, v = (torch.randn(total, h, d, generator=g, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    model, batch, policy = model_of(hq, hkv, d, "bf16"), B.Batch(cu, n_first, n_last), B.make_evict(budget, n_first, n_last)
    ws = workspace(B.earn_workspace_bytes(model, batch, 1))
    o, lse, weight = torch.empty_like(q), torch.empty(hq, total, device="cuda"), torch.empty(hkv, total, device="cuda")
    B.earn_prefill_attn(model, batch, 0, q, k, v, o, lse, ws)
    B.earn_key_weights(model, batch, 0, 16, q, k, lse, weight, ws)
    ref_w = orc.key_weights(to_np(q), to_np(k), orc.causal_attention(to_np(q), to_np(k), to_np(v), cu)[1], cu, 16)
    assert np.abs(weight.double().cpu().numpy() - ref_w).max() <= 2e-3 * ref_w.max()   # (the prefill's lse is its own: see its tolerance)
    pool = Pool(n_seq, hkv, d, "bf16", 4)
    cache = pool.cache([min(n, budget) for n in lens])
    acc = torch.zeros(n_seq, hkv, pool.cap, device="cuda")
    pos = torch.zeros(n_seq, hkv, pool.cap, dtype=torch.int32, device="cuda")
    pws = workspace(B.earn_paged_workspace_bytes(model, n_seq, cache))
    B.earn_evict_prompt_kv(model, batch, 0, policy, k, v, weight, cache, acc, pos, pws)
    torch.cuda.synchronize()
    wn, kn64, vn64 = weight.cpu().numpy(), to_np(k), to_np(v)
    state = []
    for b, n in enumerate(lens):
        heads = []
        for h in range(hkv):
            keep = orc.keep_rows(wn[h, cu[b]:cu[b + 1]], np.arange(n), budget, n_first, n_last)
            assert np.array_equal(pos[b, h, :len(keep)].cpu().numpy(), keep)
            heads.append(dict(k=[kn64[cu[b] + j, h] for j in keep], v=[vn64[cu[b] + j, h] for j in keep],
                              w=[float(wn[h, cu[b] + j]) for j in keep], pos=[int(j) for j in keep]))
        state.append(heads)
    q1 = torch.empty(n_seq, hq, d, dtype=torch.bfloat16, device="cuda")
    k1, v1 = (torch.empty(n_seq, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    o1 = torch.empty_like(q1)
    new_pos = torch.tensor(lens, dtype=torch.int32, device="cuda") - 1

    def step():
        pool.seq_len.add_(1)
        new_pos.add_(1)
        B.earn_paged_decode_attn(model, n_seq, 0, q1, k1, v1, cache, o1, acc, acc, new_pos, pos, pws)
        B.earn_evict_kv(model, n_seq, 0, policy, cache, acc, pos, acc, pos, pws)
        pool.seq_len.clamp_(max=budget)

    replay = None
    for s in range(steps):
        for t in (q1, k1, v1):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        if not graph:
            step()
        else:
            if replay is None:
                held = [x.clone() for x in (pool.seq_len, new_pos, pool.k, pool.v, acc, pos)]
                replay = torch.cuda.CUDAGraph()
                with torch.cuda.graph(replay):
                    step()
                for x, y in zip((pool.seq_len, new_pos, pool.k, pool.v, acc, pos), held):
                    x.copy_(y)
            replay.replay()
        torch.cuda.synchronize()
        ref = _reference_step(state, to_np(q1).astype(np.float64), to_np(k1), to_np(v1), [n + s for n in lens])
        err = np.abs(o1.double().cpu().numpy() - ref)
        assert err.max() <= 2e-2 and err.mean() <= 2e-3
        got_w, got_p = acc.cpu().numpy(), pos.cpu().numpy()
        for b in range(n_seq):
            for h in range(hkv):
                st = state[b][h]
                src, dst = orc.evict_moves(st["w"], st["pos"], budget, n_first, n_last)
                for x in ("k", "v", "w", "pos"):
                    for i, j in zip(src, dst):
                        st[x][j] = st[x][i]
                    del st[x][budget:]
                m = len(st["pos"])
                # (no two of these weights lie within rounding of each other, so both sides keep the same rows)
                assert np.array_equal(got_p[b, h, :m], st["pos"]), (s, b, h)
                assert np.allclose(got_w[b, h, :m], st["w"], rtol=1e-4, atol=1e-6)
    assert pool.seq_len.tolist() == [min(n + steps, budget) for n in lens]
    assert B.earn_device_status(pws) == B.EARN_OK


def test_mixed_outputs_and_a_decode_that_adds_in_place_by_graph():
    """Weights in place and positions elsewhere (and the other way round) in one eviction; a captured decode replayed on changed
    inputs, lengths among them, beside an eager call with a workspace of its own on another stream."""
    for w_here in (True, False):
        hkv, d, n = 2, 64, 40
        pool, twin = Pool(2, hkv, d, "bf16", 3), Pool(2, hkv, d, "bf16", 3)
        model, policy = model_of(hkv, hkv, d, "bf16"), B.make_evict(20, 2, 3)
        w = torch.rand(2, hkv, pool.cap, generator=gen(1), device="cuda")
        pos = torch.arange(pool.cap, dtype=torch.int32, device="cuda").expand(2, hkv, pool.cap).contiguous()
        outs = []
        for p, wo, po in ((pool, w.clone(), pos.clone()), (twin, torch.zeros_like(w), torch.zeros_like(pos))):
            cache = p.cache([n, 33])
            ws = workspace(B.earn_paged_workspace_bytes(model, 2, cache))
            wi, pi = w.clone(), pos.clone()
            if p is pool:
                wo, po = (wi, po) if w_here else (wo, pi)
            B.earn_evict_kv(model, 2, 0, policy, cache, wi, pi, wo, po, ws)
            outs.append((wo[:, :, :20], po[:, :, :20], p.k, p.v))
        for a, b in zip(*outs):
            assert torch.equal(a, b)
    hq, hkv, d = 8, 2, 128
    model, pool = model_of(hq, hkv, d, "bf16"), Pool(3, hkv, d, "bf16", 60)
    cache = pool.cache([900, 5, 60], 960)
    ws, ws2 = (workspace(B.earn_paged_workspace_bytes(model, 3, cache)) for _ in range(2))
    q = torch.randn(3, hq, d, generator=gen(2), device="cuda").to(torch.bfloat16)
    o, o2 = torch.empty_like(q), torch.empty_like(q)
    w, w2 = (torch.zeros(3, hkv, pool.cap, device="cuda") for _ in range(2))
    B.earn_paged_decode_attn(model, 3, 0, q, None, None, cache, o, w, w, None, None, ws)
    w.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.earn_paged_decode_attn(model, 3, 0, q, None, None, cache, o, w, w, None, None, ws)
    side = torch.cuda.Stream()
    for lens in ([900, 5, 60], [17, 960, 0], [1, 1, 959]):
        pool.seq_len.copy_(torch.tensor(lens, dtype=torch.int32))
        q.copy_(torch.randn(q.shape, generator=gen(sum(lens)), device="cuda"))
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            B.earn_paged_decode_attn(model, 3, 0, q, None, None, cache, o2, w2, w2, None, None, ws2)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(w, w2)


def test_two_streams_with_a_workspace_each():
    hq, hkv, d = 8, 2, 128
    model, ones = model_of(hq, hkv, d, "bf16"), []
    work = []
    for i in range(2):
        pool = Pool(4, hkv, d, "bf16", 40, seed=i)
        cache = pool.cache([600, 30, 311, 640])
        q = torch.randn(4, hq, d, generator=gen(i), device="cuda").to(torch.bfloat16)
        ws = workspace(B.earn_paged_workspace_bytes(model, 4, cache))
        work.append((pool, cache, q, ws))

    def once(pool, cache, q, ws):
        o, w = torch.empty_like(q), torch.zeros(4, hkv, pool.cap, device="cuda")
        B.earn_paged_decode_attn(model, 4, 0, q, None, None, cache, o, None, w, None, None, ws)
        return o, w

    ones = [once(*x) for x in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(20):
        got = []
        for x, s in zip(work, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(once(*x))
        torch.cuda.synchronize()
        for (o, w), (o1, w1) in zip(got, ones):
            assert torch.equal(o, o1) and torch.equal(w, w1)


# ------------------------------------------------------------------------------------------------ the session's form
def budgeted(w, budget, **kw):
    ses = make_session(w)
    b = BudgetedLayers(ses, budget, **kw)
    return ses, b


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("budget,n_last", [(10 ** 6, None), (64, None), (24, 8)])
def test_budgeted_layers(dtype, d, budget, n_last):
    """A model of two full layers through the session: with a budget nothing reaches, every decode output is that of the whole
    cache; with a small one the outputs are the oracle's over the rows that `pos` names, and no more rows are held."""
    w = wl.Workload("budget", batch=3, n_layers=2, split_k=2, n_q_heads=4, n_kv_heads=2, head_dim=d, dtype=dtype, prompt_len=0,
                    lens=(90, 40, 131), r_head=4, r_tail=4, decode_steps=6, seed=51)
    cu, lens = wl.cu_seqlens(w), wl.seqlens(w)
    ses, bud = budgeted(w, budget, n_last=n_last, paged_shuffle_seed=3)
    rows = []      # per layer and sequence: every token's key and value so far
    for layer in range(2):
        q, k, v = wl.layer_qkv(w, layer, "cuda")
        lse = torch.empty(w.n_q_heads, int(cu[-1]), device="cuda")
        ses.prefill_layer(layer, q, k, v, lse=lse)
        bud.take_prompt(layer, q, k, v, lse)
        rows.append([[list(to_np(x)[cu[b]:cu[b + 1]]) for x in (k, v)] for b in range(w.batch)])
    for step in range(1, w.decode_steps + 1):
        bud.begin_step()
        for layer in range(2):
            before = bud.pos[layer].cpu().numpy()
            n_before = [min(int(n) + step - 1, budget) for n in lens]
            q, k, v = wl.decode_qkv(w, layer, step, "cuda")
            o = bud.decode_layer(layer, q, k, v)
            if budget >= 10 ** 6:
                whole = ses.decode_layer(layer, step, q, k, v)
                assert_close(o, to_np(whole).astype(np.float64), dtype, "whole cache")
            for b in range(w.batch):
                for x, new in zip(rows[layer][b], (k, v)):
                    x.append(to_np(new)[b])
                ref = np.zeros((w.n_q_heads, d))
                for h in range(2):
                    idx = list(before[b, h, :n_before[b]]) + [len(rows[layer][b][0]) - 1]
                    kk, vv = (np.asarray(x)[idx, h][:, None] for x in rows[layer][b])
                    ref[2 * h:2 * h + 2] = orc.paged_decode(to_np(q)[b, 2 * h:2 * h + 2], kk, vv)[0]
                assert_close(o[b], ref, dtype, f"step {step} layer {layer} sequence {b}")
        bud.end_step()
        assert bud.seq_len.tolist() == [min(int(n) + step, budget) for n in lens]
        for layer in range(2):     # the registers and the last rows are there, and no token twice
            p = bud.pos[layer].cpu().numpy()
            for b in range(w.batch):
                m = int(bud.seq_len[b])
                for h in range(2):
                    held = set(p[b, h, :m].tolist())
                    assert len(held) == m and set(range(w.r_head)) <= held
                    total = int(lens[b]) + step
                    assert set(range(total - (w.r_tail if n_last is None else n_last), total)) <= held
    assert bud.device_status() == B.EARN_OK
    with pytest.raises(ValueError, match="one beam"):
        BudgetedLayers(make_session(w.replace(beams=2)), 16)


def test_budgeted_layers_refuse_steps_without_room():
    """Below the budget a session has room for max_new tokens; at the budget there is no end; without full layers nothing to do."""
    w = wl.Workload("budget", batch=2, n_layers=2, split_k=1, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", prompt_len=0,
                    lens=(20, 9), r_head=2, r_tail=2, decode_steps=3, seed=1)
    _, wide = budgeted(w, 100)
    _, tight = budgeted(w, 16)
    for _ in range(3):
        wide.begin_step()
    with pytest.raises(ValueError, match="no room"):
        wide.begin_step()
    assert wide.seq_len.tolist() == [23, 12]
    for _ in range(9):
        tight.begin_step()
        tight.end_step()
    assert tight.seq_len.tolist() == [16, 16]
    _, none = budgeted(w.replace(split_k=0), 16)
    assert none.device_status() == B.EARN_OK


def test_binding_refusals_on_the_device():
    """What the wrappers turn down before the library is called: another type, a strided view, too few elements, host memory."""
    hq, hkv, d = 4, 2, 128
    pool = Pool(2, hkv, d, "bf16", 2)
    cache = pool.cache([5, 9])
    model = model_of(hq, hkv, d, "bf16")
    ws = workspace(B.earn_paged_workspace_bytes(model, 2, cache))
    q = torch.zeros(2, hq, d, device="cuda", dtype=torch.bfloat16)
    n0 = B.earn_launch_count()
    for bad in (q.float(), torch.zeros(2, d, hq, device="cuda", dtype=torch.bfloat16).transpose(1, 2), q[:1], q.cpu()):
        with pytest.raises(ValueError, match="q: "):
            B.earn_paged_decode_attn(model, 2, 0, bad, None, None, cache, q, workspace=ws)
    with pytest.raises(ValueError, match="weight_out"):
        B.earn_paged_decode_attn(model, 2, 0, q, None, None, cache, q, weight_out=torch.zeros(2, hkv, 8, device="cuda"), workspace=ws)
    with pytest.raises(ValueError, match="fewer than 3"):
        B.earn_paged_decode_attn(model, 3, 0, q, None, None, cache, q, workspace=ws)
    with pytest.raises(ValueError, match="cache of"):
        B.earn_paged_decode_attn(model_of(hq, hkv, 64, "bf16"), 2, 0, q, None, None, cache, q, workspace=ws)
    with pytest.raises(B.EarnError):
        B.earn_paged_decode_attn(model, 2, 0, q, None, None, cache, q, workspace=None)
    assert B.earn_launch_count() == n0
