"""How exact the key weights are in the mean, where the elementwise bounds of the other tests leave room for a bias: against the
64-bit definition over long windows, and against the prefill's own denominators, under which every query hands out exactly one."""
import numpy as np
import pytest
import torch

from paper_2507_00715_b200 import binding as B

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(n, hq, hkv, d, dtype, spread, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q = (spread * torch.randn(n, hq, d, generator=g, device="cuda")).to(DT[dtype])
    return q, torch.randn(n, hkv, d, generator=g, device="cuda").to(DT[dtype])


def call(q, k, lse, scale, dtype, n_obs):
    n, hq, d = q.shape
    model = B.make_model(1, 1, hq, k.shape[1], d, dtype, scale)
    batch = B.Batch(np.asarray([0, n], np.int32), 0, 0)
    ws = torch.empty(B.earn_workspace_bytes(model, batch, 1), dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(ws)
    if lse is None:
        lse = torch.empty(hq, n, device="cuda")
        B.earn_prefill_attn(model, batch, 0, q, k, torch.zeros_like(k), torch.empty_like(q), lse, ws)
    w = torch.empty(k.shape[1], n, device="cuda")
    B.earn_key_weights(model, batch, 0, n_obs, q, k, lse, w, ws)
    assert B.earn_device_status(ws) == B.EARN_OK
    return w


def logits(q, k, h, scale, a, e):
    """fp64 [e, e - a]: keys 0 .. e - 1 under the queries a .. e - 1 of head h, those a query does not see -inf."""
    s = k[:e, h * k.shape[1] // q.shape[1]].double() @ q[a:e, h].double().T * (scale or q.shape[2] ** -0.5)
    later = torch.arange(e, device="cuda")[:, None] > torch.arange(a, e, device="cuda")[None, :]
    return s.masked_fill_(later, float("-inf"))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("scale", [0.0, 0.05])
def test_mean_error_over_a_long_window(d, scale):
    """4096 rows, every query, a group of four, logits of at most unit variance: relative error over all weights (root of the
    sums of squares) and its signed mean.  The mean error of a logit under the softmax weights: each of the D / 16 steps of the
    matrix unit truncates the sum so far, half a unit (2^-24) in the mean, and the sum so far grows as a random walk: 2/3 D/16
    2^-24.  Scale and scale times log2 e: 2 * 2^-24.  Exponential unit: 2^-22.  The roundings of single arguments average out."""
    n, hq, hkv = 4096, 8, 2
    q, k = inputs(n, hq, hkv, d, "bf16", 1.0, seed=d)
    lse = torch.empty(hq, n, device="cuda")
    ref = torch.zeros(hkv, n, dtype=torch.float64, device="cuda")
    for h in range(hq):
        for a in range(0, n, 1024):
            s = logits(q, k, h, scale, a, a + 1024)
            lse[h, a:a + 1024] = torch.logsumexp(s, 0).float()
            ref[h * hkv // hq, :a + 1024] += torch.exp(s - lse[h, a:a + 1024].double()).sum(1)
    err = call(q, k, lse, scale, "bf16", n).double() - ref
    tol = 2.0 ** -22 + 2 / 3 * d / 16 * 2.0 ** -24 + 2 * 2.0 ** -24
    assert float(err.norm() / ref.norm()) <= tol, (float(err.norm() / ref.norm()), tol)
    assert abs(float(err.sum() / ref.sum())) <= tol, (float(err.sum() / ref.sum()), tol)


@pytest.mark.parametrize("scale", [0.0, 0.1, 0.03])
@pytest.mark.parametrize("n_obs", [4096, 64])
def test_every_query_hands_out_one_under_the_prefills_denominators(scale, n_obs):
    """Logits of a standard deviation of 6, where a scale that differs from the prefill's shows most: the weights of a kv head sum
    to (queries) x (heads of the group).  Both kernels take the same products and the same scale, so what is left is systematic
    at most in the exponential unit (2^-22 in each) and in the logarithm of the prefill's sum (2^-22), and 2^-23 for the rest (log2 e and
    ln 2 in 32 bits: 1.6e-8 of a denominator of 24 is 4e-7 in the window's few rows, but log2 e is taken in two parts: 2.7e-9)."""
    n, hq, hkv, d = 4096, 8, 2, 128
    q, k = inputs(n, hq, hkv, d, "bf16", 6.0 * d ** -0.5 / (scale or d ** -0.5), seed=int(1000 * scale) + n_obs)
    w = call(q, k, None, scale, "bf16", n_obs)
    got = w.double().sum(1) / (n_obs * (hq // hkv)) - 1.0
    assert float(got.abs().max()) <= 3 * 2.0 ** -22 + 2.0 ** -23, got.tolist()


@pytest.mark.parametrize("dtype,depth", [("f32", 2 + 16 + 64 + 4), ("bf16", 32 + 512 + 4)])
def test_small_terms_of_a_long_window_are_not_lost(dtype, depth):
    """The first eight queries give 1 each, 8184 others 2^-22.5 each (zero queries, denominators to match), under eight heads: a
    sum that took them one by one would lose every one of the small ones, 1.7e-4 of the weight.  A sum of positive terms is off
    by at most 2^-24 per addition that a term goes through.  fp32: 64 columns of a tile, four of them a thread's (2 additions),
    16 tiles, 64 sixteens of tiles, 16 threads (4).  bf16: half of a tile's 64 columns, 512 tiles, and the four parts of a key's sum."""
    n, g, d = 8192, 8, 64
    q, k = inputs(n, g, 1, d, dtype, 0.0, seed=1)
    lse = torch.full((g, n), 22.5 * np.log(2.0), device="cuda")
    lse[:, :8] = 0.0
    w = call(q, k, lse, 0.0, dtype, n)
    seen = torch.arange(n, 0, -1, device="cuda").double()             # queries that see key j
    large = (8.0 - torch.arange(n, device="cuda").double()).clamp_(min=0.0)
    ref = g * (large + (seen - large) * torch.exp(-lse[0, -1].double()))
    err = ((w[0].double() - ref).abs() / ref)
    # a small term itself: 22.5 (two roundings, log2 e) and the exponential unit
    tol = torch.full_like(ref, depth * 2.0 ** -24 + 22.5 * 3 * 2.0 ** -24 + 2.0 ** -22)
    tol[:8] = depth * 2.0 ** -24 + 2.0 ** -22
    assert bool((err <= tol).all()), (float(err[:8].max()), float(err.max()))
