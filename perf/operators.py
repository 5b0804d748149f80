"""The operators of an evictable key-value cache, as a user's program calls them: cases, inputs, plain forms.

A full layer's cache (a layer in front of the split, which keeps every prompt row) can be held to a budget of rows per
sequence and kv head.  Four operators make that up:

  key_weights   the attention weight every prompt row has received from the last n_obs queries of its sequence, summed
                over those queries and over the query heads of a kv head (from the prefill's softmax denominators);
  evict_prompt  the budget's worth of prompt rows per kv head -- the first n_first, the last n_last, and of the others
                those with the most weight -- copied from the packed prompt into a paged cache, in order of position;
  paged_decode  one new token per sequence: its K/V row is appended to the pages, its queries attend over the whole
                paged list, and what each row received is added to the row's accumulated weight;
  evict_rows    the cache in place, from its present length down to the budget: kept rows that lie behind the budget
                move into the places of rows that go, in order.

With ``own`` false ``run`` computes an operator with elementary torch operations in 32 bits; with ``own`` true it makes
the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 16
HEADS = ((4, 4, 64), (12, 2, 128), (32, 8, 128), (28, 4, 128), (32, 32, 128), (8, 1, 64), (16, 4, 64), (20, 4, 128))
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------- cases
def listed():
    def case(name, op, batch, heads, dtype, len_lo, len_hi, **kw):
        return dict(name=name, op=op, batch=batch, hq=heads[0], hkv=heads[1], d=heads[2], dtype=dtype, len_lo=len_lo,
                    len_hi=len_hi, **kw)

    tiny, small, base, gqa7 = (4, 4, 64), (12, 2, 128), (32, 8, 128), (28, 4, 128)
    return [
        # one short prompt in fp32 (the debugging workload), weights from its four tail registers and four rows more
        case("weights-one-prompt-f32", "key_weights", 1, tiny, "f32", 256, 256, n_obs=8),
        # a ragged serving batch whose rows are weighed by the last 32 queries (registers included)
        case("weights-window-ragged", "key_weights", 128, base, "bf16", 128, 2048, n_obs=32),
        # long histories weighed by every query of the prompt
        case("weights-whole-long", "key_weights", 8, base, "bf16", 4096, 4096, n_obs=4096),
        # the debugging workload's prompt cut to a quarter
        case("prompt-one-f32", "evict_prompt", 1, tiny, "f32", 256, 256, budget=64, n_first=4, n_last=4),
        # the ragged batch held to 512 rows a head, some prompts shorter than that
        case("prompt-ragged", "evict_prompt", 128, base, "bf16", 128, 2048, budget=512, n_first=16, n_last=32),
        # very long histories cut to an eighth
        case("prompt-long", "evict_prompt", 8, base, "bf16", 12000, 16384, budget=2048, n_first=16, n_last=64),
        # a single user's next token, where latency counts; no weights kept
        case("decode-one", "paged_decode", 1, small, "bf16", 512, 512, weigh=False),
        # odd group size, short lists of uneven length
        case("decode-short-ragged", "paged_decode", 48, gqa7, "bf16", 50, 200, weigh=True),
        # the ordinary serving batch
        case("decode-batch", "paged_decode", 64, base, "bf16", 700, 1044, weigh=True),
        # a few long caches: the list is split over the GPU and joined
        case("decode-long", "paged_decode", 8, base, "bf16", 20000, 32768, weigh=True),
        # the serving batch at its budget: every step one row too many
        case("evict-step", "evict_rows", 64, base, "bf16", 1025, 1025, budget=1024, n_first=16, n_last=64),
        # long caches halved at once when memory runs short
        case("evict-half", "evict_rows", 8, base, "bf16", 8192, 8192, budget=4096, n_first=16, n_last=64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("key_weights", "evict_prompt", "paged_decode", "evict_rows"))
    hq, hkv, d = rng.choice(HEADS)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    batch = _log_int(rng, 1, 128)
    most = {"key_weights": 8192, "evict_prompt": 16384, "paged_decode": 32768, "evict_rows": 16384}[op]
    len_hi = _log_int(rng, 1, most)
    len_lo = len_hi if rng.random() < 0.3 else rng.randint(1, len_hi)
    case = dict(op=op, batch=batch, hq=hq, hkv=hkv, d=d, dtype=dtype, len_lo=len_lo, len_hi=len_hi)
    if op == "key_weights":
        case["n_obs"] = _log_int(rng, 1, len_hi)
        costs = lambda: case["batch"] * hq * d * len_hi * min(case["n_obs"], len_hi) * (8 if dtype == "f32" else 1)  # noqa: E731
        limit = 8 * 32 * 128 * 4096 * 4096 // 2
    else:
        # (rows of the cache, with the plain form's 32-bit copies of them in mind)
        costs = lambda: case["batch"] * hkv * d * len_hi * (2 if dtype == "f32" else 1)  # noqa: E731
        limit = 8 * 8 * 128 * {"evict_prompt": 14000, "paged_decode": 26000, "evict_rows": 8192}[op]
    while case["batch"] > 1 and costs() > limit:
        case["batch"] = case["batch"] // 2
    if op == "key_weights":
        while costs() > limit:
            case["n_obs"] = max(1, case["n_obs"] // 2)
    else:
        while costs() > limit:
            len_hi = len_hi // 2
            case["len_hi"], case["len_lo"] = len_hi, min(len_lo, len_hi)
    if op == "paged_decode":
        case["weigh"] = rng.random() < 0.7
    elif op != "key_weights":
        budget = _log_int(rng, 1, max(1, int(case["len_hi"] * 1.1)))
        case["budget"] = budget
        case["n_first"] = rng.randint(0, min(budget, 16))
        case["n_last"] = rng.randint(0, min(budget - case["n_first"], 64))
    return case


def _lens(case):
    """The sequences' lengths: spread over [len_lo, len_hi], the same for every seed, the longest among them."""
    lo, hi, n = case["len_lo"], case["len_hi"], case["batch"]
    return [hi - int((hi - lo + 1) * ((i * 0.6180339887498949) % 1.0)) if hi > lo else hi for i in range(n)]


# ---------------------------------------------------------------------------------------------------- inputs
def _prompt_qkv(case, lens, g, want):
    """Packed rows, N(0,1), with the pull towards the first and the last row of a prompt that trained models show."""
    d, hq, hkv, total = case["d"], case["hq"], case["hkv"], sum(lens)
    kw = dict(generator=g, device="cuda", dtype=torch.float32)
    u = torch.randn(hkv, d, **kw)
    u = u / u.norm(dim=-1, keepdim=True)
    out = {}
    dt = DTYPES[case["dtype"]]
    if "q" in want:
        q = torch.randn(total, hkv, hq // hkv, d, **kw)
        out["q"] = (q + math.sqrt(d) * u[:, None]).reshape(total, hq, d).to(dt)
    if "k" in want:
        k = torch.randn(total, hkv, d, **kw)
        ends = torch.tensor(lens, device="cuda").cumsum(0)
        starts = ends - torch.tensor(lens, device="cuda")
        k[starts] += 4.0 * u
        k[ends - 1] += 4.0 * u
        out["k"] = k.to(dt)
    if "v" in want:
        out["v"] = torch.randn(total, hkv, d, **kw).to(dt)
    return out


def _weights(shape, g):
    """Accumulated attention weights: a long tail, rows that nobody ever looked at (exact zeros), and equal values."""
    w = torch.exp(2.0 * torch.randn(shape, generator=g, device="cuda")) * 0.05
    pick = torch.rand(shape, generator=g, device="cuda")
    w = torch.where(pick < 0.1, torch.zeros_like(w), w)
    return torch.where(pick > 0.9, (w * 8.0).round() * 0.125, w)


def _pages(case, n_rows_cap, g):
    per_seq = -(-n_rows_cap // PAGE)
    n_pages = case["batch"] * per_seq
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).reshape(case["batch"], per_seq)
    return per_seq, n_pages, table


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    lens = _lens(case)
    st = {"case": dict(case), "lens": lens, "scale": 1.0 / math.sqrt(case["d"])}
    st["len_dev"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    st["cu"] = cu
    st["cu_dev"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    b, hq, hkv, d, dt = case["batch"], case["hq"], case["hkv"], case["d"], DTYPES[case["dtype"]]
    if case["op"] == "key_weights":
        st.update(_prompt_qkv(case, lens, g, "qk"))
        # the softmax denominators that the prefill leaves (needed for the rows of the window)
        lse = torch.zeros(hq, cu[-1], device="cuda")
        for i, n in enumerate(lens):
            lo, hi, m = cu[i], cu[i + 1], min(case["n_obs"], n)
            k = st["k"][lo:hi].float().repeat_interleave(hq // hkv, 1).permute(1, 2, 0)
            for a in range(n - m, n, 1024):
                e = min(n, a + 1024)
                s = torch.matmul(st["q"][lo + a:lo + e].float().permute(1, 0, 2), k) * st["scale"]
                hidden = torch.arange(n, device="cuda")[None, :] > torch.arange(a, e, device="cuda")[:, None]
                lse[:, lo + a:lo + e] = torch.logsumexp(s.masked_fill_(hidden, float("-inf")), -1)
        st["lse"] = lse
        st["weight"] = torch.empty(hkv, cu[-1], device="cuda")
    elif case["op"] == "evict_prompt":
        st.update(_prompt_qkv(case, lens, g, "kv"))
        st["weight"] = _weights((hkv, cu[-1]), g)
        st["per_seq"], st["n_pages"], st["table"] = _pages(case, case["budget"], g)
        cap = st["per_seq"] * PAGE
        st["k_pages"] = torch.zeros(st["n_pages"], PAGE, hkv, d, device="cuda", dtype=dt)
        st["v_pages"] = torch.zeros_like(st["k_pages"])
        st["weight_out"] = torch.zeros(b, hkv, cap, device="cuda")
        st["pos_out"] = torch.zeros(b, hkv, cap, device="cuda", dtype=torch.int32)
    else:
        st["per_seq"], st["n_pages"], st["table"] = _pages(case, case["len_hi"] + (case["batch"] % 3) * PAGE, g)
        cap = st["per_seq"] * PAGE
        rows = _prompt_qkv(dict(case, batch=1), [st["n_pages"] * PAGE], g, "kv")
        st["k_pages"] = rows["k"].reshape(st["n_pages"], PAGE, hkv, d)
        st["v_pages"] = rows["v"].reshape(st["n_pages"], PAGE, hkv, d)
        if case["op"] == "paged_decode":
            st["q"] = (1.5 * torch.randn(b, hq, d, generator=g, device="cuda")).to(dt)
            st["k_new"] = torch.randn(b, hkv, d, generator=g, device="cuda").to(dt)
            st["v_new"] = torch.randn(b, hkv, d, generator=g, device="cuda").to(dt)
            st["o"] = torch.empty_like(st["q"])
            if case["weigh"]:
                st["weight"] = _weights((b, hkv, cap), g)
                st["weight_out"] = torch.zeros(b, hkv, cap, device="cuda")
                st["pos"] = torch.zeros(b, hkv, cap, device="cuda", dtype=torch.int32)
                st["new_pos"] = torch.randint(0, 1 << 20, (b,), generator=g, device="cuda").to(torch.int32)
        else:
            # the positions a head's rows came from: its slots hold distinct tokens, in order but for a few refilled ones
            st["weight"] = _weights((b, hkv, cap), g)
            pos = torch.arange(cap, device="cuda", dtype=torch.int32).expand(b, hkv, cap).contiguous()
            n = min(cap, case["len_lo"])
            if n > 4:
                i, j = torch.randint(0, n, (2,), generator=g, device="cuda").unbind()
                pos[:, :, torch.stack((i, j))] = pos[:, :, torch.stack((j, i))]
            st["pos"] = pos
            st["weight_out"] = torch.zeros(b, hkv, cap, device="cuda")
            st["pos_out"] = torch.zeros(b, hkv, cap, device="cuda", dtype=torch.int32)
    return st


# ---------------------------------------------------------------------------------------------------- plain forms
def _rows_of(st, n):
    """Row numbers of list positions 0 .. n - 1 of every sequence in the page pool: [B, n]."""
    j = torch.arange(n, device="cuda")
    return st["table"].long()[:, j // PAGE] * PAGE + j % PAGE


def _plain_key_weights(st):
    c, out = st["case"], st["weight"]
    hkv, grp = c["hkv"], c["hq"] // c["hkv"]
    for i, n in enumerate(st["lens"]):
        lo, m = st["cu"][i], min(c["n_obs"], n)
        k = st["k"][lo:lo + n].float().permute(1, 2, 0)                                        # [Hkv, D, n]
        q = st["q"][lo + n - m:lo + n].float().reshape(m, hkv, grp, c["d"]).permute(1, 2, 0, 3)  # [Hkv, g, m, D]
        s = torch.matmul(q.reshape(hkv, grp * m, c["d"]), k).reshape(hkv, grp, m, n)
        s = s * st["scale"] - st["lse"][:, lo + n - m:lo + n].reshape(hkv, grp, m, 1)
        seen = torch.arange(n, device="cuda")[None, :] <= torch.arange(n - m, n, device="cuda")[:, None]
        out[:, lo:lo + n] = torch.where(seen, torch.exp(s), torch.zeros_like(s)).sum((1, 2))
    return {"weight": out}


def _keep(weight, pos, valid, last, budget, n_first, n_last):
    """Which rows stay: [B, Hkv, n].  Rank by (protected first, more weight first, lower row first)."""
    safe = (pos < n_first) | (pos > last - n_last)
    w = torch.nan_to_num(weight, nan=float("-inf"), posinf=float("inf"), neginf=float("-inf"))
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    by = torch.where(valid, torch.where(safe, 0, 1), 2).gather(-1, order)
    order = order.gather(-1, torch.sort(by, dim=-1, stable=True).indices)
    rank = torch.empty_like(order).scatter_(-1, order, torch.arange(order.shape[-1], device="cuda").expand_as(order).contiguous())
    return valid & (rank < budget)


def _plain_evict_prompt(st):
    c, hkv = st["case"], st["case"]["hkv"]
    n = max(st["lens"])
    lens = st["len_dev"].long()
    j = torch.arange(n, device="cuda")
    valid = (j[None, :] < lens[:, None])[:, None, :].expand(-1, hkv, -1)
    src = torch.minimum(st["cu_dev"][:-1].long()[:, None] + j[None, :], torch.tensor(st["cu"][-1] - 1, device="cuda"))
    weight = st["weight"][:, src].permute(1, 0, 2)                                           # [B, Hkv, n]
    keep = _keep(weight, j.expand_as(weight), valid, (lens - 1)[:, None, None], c["budget"], c["n_first"], c["n_last"])
    bi, hi, ji = keep.nonzero(as_tuple=True)
    slot = (keep.cumsum(-1) - 1)[bi, hi, ji]
    row = _rows_of(st, c["budget"])[bi, slot]
    d = c["d"]
    st["k_pages"].view(-1, hkv, d)[row, hi] = st["k"][src[bi, ji], hi]
    st["v_pages"].view(-1, hkv, d)[row, hi] = st["v"][src[bi, ji], hi]
    st["weight_out"][bi, hi, slot] = weight[bi, hi, ji]
    st["pos_out"][bi, hi, slot] = ji.to(torch.int32)
    return {"k": st["k_pages"], "v": st["v_pages"], "weight": st["weight_out"], "pos": st["pos_out"]}


def _plain_paged_decode(st):
    c = st["case"]
    b, hkv, grp, d, n = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["d"], max(st["lens"])
    lens = st["len_dev"].long()
    rows = _rows_of(st, n)
    newest = rows.gather(1, (lens - 1)[:, None])[:, 0]
    k_rows, v_rows = st["k_pages"].view(-1, hkv, d), st["v_pages"].view(-1, hkv, d)
    k_rows[newest] = st["k_new"]
    v_rows[newest] = st["v_new"]
    q = st["q"].float().reshape(b, hkv, grp, d)
    s = torch.matmul(q, k_rows[rows].permute(0, 2, 3, 1).float()) * st["scale"]               # [B, Hkv, g, n]
    seen = (torch.arange(n, device="cuda")[None, :] < lens[:, None])[:, None, None, :]
    s = s.masked_fill(~seen, float("-inf"))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    o = torch.matmul(p, v_rows[rows].permute(0, 2, 1, 3).float())
    out = {"o": o.reshape(b, c["hq"], d).to(st["q"].dtype), "k": st["k_pages"], "v": st["v_pages"]}
    if c["weigh"]:
        got = p.sum(2)                                                                       # [B, Hkv, n]
        fresh = (torch.arange(n, device="cuda")[None, :] == (lens - 1)[:, None])[:, None, :]
        new = torch.where(fresh, got, st["weight"][:, :, :n] + got)
        st["weight_out"][:, :, :n] = torch.where(seen[:, 0], new, st["weight_out"][:, :, :n])
        st["pos"].scatter_(2, (lens - 1)[:, None, None].expand(b, hkv, 1), st["new_pos"][:, None, None].expand(b, hkv, 1))
        out["weight"], out["pos"] = st["weight_out"], st["pos"]
    return out


def _plain_evict_rows(st):
    c, hkv, d = st["case"], st["case"]["hkv"], st["case"]["d"]
    cap, lens, budget = st["per_seq"] * PAGE, st["len_dev"].long()[:, None, None], st["case"]["budget"]
    j = torch.arange(cap, device="cuda").expand(c["batch"], hkv, cap)
    valid = j < lens
    last = torch.where(valid, st["pos"], -1).amax(-1, keepdim=True)
    keep = _keep(st["weight"], st["pos"], valid, last, budget, c["n_first"], c["n_last"])
    bi, hi, jd = ((j < torch.clamp(lens, max=budget)) & ~keep).nonzero(as_tuple=True)   # places that fall free, in order
    _, _, js = ((j >= budget) & keep).nonzero(as_tuple=True)                             # rows that move there, in order
    rows = _rows_of(st, cap)
    for pages in (st["k_pages"].view(-1, hkv, d), st["v_pages"].view(-1, hkv, d)):
        pages[rows[bi, jd], hi] = pages[rows[bi, js], hi]
    left = j < torch.clamp(lens, max=budget)
    for name in ("weight", "pos"):
        out = torch.where(left, st[name], st[name + "_out"])
        out[bi, hi, jd] = st[name][bi, hi, js]
        st[name + "_out"] = out
    return {"k": st["k_pages"], "v": st["v_pages"], "weight": st["weight_out"], "pos": st["pos_out"]}


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _handles(st):
    """What a program keeps beside its tensors: the model and batch descriptions, the cache and the workspace."""
    import numpy as np

    from paper_2507_00715_b200 import binding as B

    c = st["case"]
    h = {"B": B, "model": B.make_model(1, 1, c["hq"], c["hkv"], c["d"], c["dtype"])}
    if c["op"] in ("key_weights", "evict_prompt"):
        h["batch"] = B.Batch(np.asarray(st["cu"], dtype=np.int32), 0, 0, cu_seqlens_dev=st["cu_dev"])
    if c["op"] == "key_weights":
        need = B.earn_workspace_bytes(h["model"], h["batch"], 1)
    else:
        h["cache"] = B.make_paged_cache(st["k_pages"], st["v_pages"], st["table"], st["len_dev"],
                                        max_len=c["budget"] if c["op"] == "evict_prompt" else c["len_hi"])
        need = B.earn_paged_workspace_bytes(h["model"], c["batch"], h["cache"])
    if "budget" in c:
        h["policy"] = B.make_evict(c["budget"], c["n_first"], c["n_last"])
    h["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    B.earn_workspace_init(h["workspace"])
    return h


def _own_call(st):
    if "handles" not in st:
        st["handles"] = _handles(st)
    h, c = st["handles"], st["case"]
    B = h["B"]
    if c["op"] == "key_weights":
        B.earn_key_weights(h["model"], h["batch"], 0, c["n_obs"], st["q"], st["k"], st["lse"], st["weight"], h["workspace"])
        return {"weight": st["weight"]}
    if c["op"] == "evict_prompt":
        B.earn_evict_prompt_kv(h["model"], h["batch"], 0, h["policy"], st["k"], st["v"], st["weight"], h["cache"],
                               st["weight_out"], st["pos_out"], h["workspace"])
    elif c["op"] == "paged_decode":
        B.earn_paged_decode_attn(h["model"], c["batch"], 0, st["q"], st["k_new"], st["v_new"], h["cache"], st["o"],
                                 st.get("weight"), st.get("weight_out"), st.get("new_pos"), st.get("pos"), h["workspace"])
        out = {"o": st["o"], "k": st["k_pages"], "v": st["v_pages"]}
        return dict(out, weight=st["weight_out"], pos=st["pos"]) if c["weigh"] else out
    else:
        B.earn_evict_kv(h["model"], c["batch"], 0, h["policy"], h["cache"], st["weight"], st["pos"], st["weight_out"],
                        st["pos_out"], h["workspace"])
    return {"k": st["k_pages"], "v": st["v_pages"], "weight": st["weight_out"], "pos": st["pos_out"]}


def run(state):
    if own:
        return _own_call(state)
    return {"key_weights": _plain_key_weights, "evict_prompt": _plain_evict_prompt, "paged_decode": _plain_paged_decode,
            "evict_rows": _plain_evict_rows}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------- necessary work
def work(case):
    lens, hq, hkv, d = _lens(case), case["hq"], case["hkv"], case["d"]
    e = 4 if case["dtype"] == "f32" else 2
    kv_row = 2 * hkv * d * e
    if case["op"] == "key_weights":
        seen = sum(m * (n - m) + m * (m + 1) // 2 for n in lens for m in (min(case["n_obs"], n),))
        window = sum(min(case["n_obs"], n) for n in lens)
        return {"bytes": window * hq * (d * e + 4) + sum(lens) * hkv * (d * e + 4), "flops": 2 * hq * d * seen}
    if case["op"] == "evict_prompt":
        kept = sum(min(case["budget"], n) for n in lens)
        return {"bytes": sum(lens) * hkv * 4 + kept * (2 * kv_row + hkv * 8), "flops": sum(lens) * hkv}
    if case["op"] == "paged_decode":
        rows, b = sum(lens), case["batch"]
        return {"bytes": rows * (kv_row + (hkv * 8 if case["weigh"] else 0)) + b * (2 * hq * d * e + kv_row),
                "flops": 4 * hq * d * rows}
    # evict_rows: a row behind the budget is among the kept ones as often as any other (the protected ones aside)
    moved = sum((n - case["budget"]) * case["budget"] // n for n in lens if n > case["budget"])
    left = sum(min(n, case["budget"]) for n in lens)
    return {"bytes": sum(lens) * hkv * 8 + left * hkv * 8 + moved * 2 * kv_row, "flops": sum(lens) * hkv}


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The computed outputs (weights of the prompt's rows; a decode step's output and weights) by their definitions in
    64 bits.  The two evictions move rows and compute nothing."""
    if case["op"] not in ("key_weights", "paged_decode"):
        return None
    st = prepare(case, seed)
    hq, hkv, scale = case["hq"], case["hkv"], 1.0 / math.sqrt(case["d"])
    grp = hq // hkv
    if case["op"] == "key_weights":
        out = torch.zeros(hkv, st["cu"][-1], dtype=torch.float64, device="cuda")
        for i, n in enumerate(st["lens"]):
            lo, first = st["cu"][i], n - min(case["n_obs"], n)
            for h in range(hq):
                key = st["k"][lo:lo + n, h // grp].double()
                for a in range(first, n, 2048):
                    e = min(n, a + 2048)
                    logit = key[:e] @ (st["q"][lo + a:lo + e, h].double() * scale).T       # [keys, queries]
                    w = torch.exp(logit - st["lse"][h, lo + a:lo + e].double())
                    later = torch.arange(e, device="cuda")[:, None] > torch.arange(a, e, device="cuda")[None, :]
                    w[later] = 0.0
                    out[h // grp, lo:lo + e] += w.sum(1)
        return {"weight": out}
    o = torch.zeros(case["batch"], hq, case["d"], dtype=torch.float64, device="cuda")
    weight = st["weight_out"].double() if case["weigh"] else None
    for i, n in enumerate(st["lens"]):
        page = st["table"][i].long()
        key = st["k_pages"][page].flatten(0, 1)[:n].double()
        val = st["v_pages"][page].flatten(0, 1)[:n].double()
        key[n - 1], val[n - 1] = st["k_new"][i].double(), st["v_new"][i].double()
        if case["weigh"]:
            weight[i, :, :n - 1] = st["weight"][i, :, :n - 1].double()
        for h in range(hq):
            a = torch.softmax(key[:, h // grp] @ st["q"][i, h].double() * scale, 0)
            o[i, h] = a @ val[:, h // grp]
            if case["weigh"]:
                weight[i, h // grp, :n] += a
    out = {"o": o, "k": None, "v": None}
    return dict(out, weight=weight, pos=None) if case["weigh"] else out
