"""The operators of a step of several new tokens over a paged cache, as a user's program calls them: cases, inputs, plain forms.

A full layer's cache lives in pages of 16 rows.  A step brings every sequence to a target length: some grow by one token,
some by a chunk of a prompt or a drafted continuation, some are cut back or end.  Three operators make that up:

  page_tables   from the lengths held and the target lengths: pages given back, pages taken, block tables, the offsets of
                the new tokens in the packed batch, and every new token's position and slot in the page pool;
  rope          rotary positions: the rows of Q and K turned by their tokens' positions, dense (a prompt, or the gradient of
                one), or with K and V appended to the pages by slot;
  chunk_attn    causal attention of every sequence's new tokens over its whole paged list.

With ``own`` false ``run`` computes an operator with elementary torch operations in 32 bits (angles in 64); with ``own`` true
it makes the framework's calls.
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
    def tables(name, n_seq, len_hi, per_seq, free, **shares):
        return dict(name=name, op="page_tables", n_seq=n_seq, len_hi=len_hi, per_seq=per_seq, free=free, **shares)

    def rope(name, form, tokens, heads, dtype, rot, layout, far):
        return dict(name=name, op="rope", form=form, tokens=tokens, hq=heads[0], hkv=heads[1], d=heads[2], dtype=dtype, rot=rot,
                    layout=layout, far=far)

    def chunk(name, batch, heads, dtype, old, new, singles, lse):
        return dict(name=name, op="chunk_attn", batch=batch, hq=heads[0], hkv=heads[1], d=heads[2], dtype=dtype, old_lo=old[0],
                    old_hi=old[1], new_lo=new[0], new_hi=new[1], singles=singles, lse=lse)

    tiny, small, base, gqa7 = (4, 4, 64), (12, 2, 128), (32, 8, 128), (28, 4, 128)
    return [
        # the serving batch's step: one more token each, a page now and then
        tables("tables-step", 64, 1044, 128, 1.0, grow=0.0, end=0.0, cut=0.0, chunk=1),
        # a busy server: single tokens, chunks of prompts, drafts cut back, requests that end; hardly enough free pages
        tables("tables-mixed", 512, 2048, 160, 0.9, grow=0.25, end=0.1, cut=0.2, chunk=256),
        # a ragged batch of prompts taken whole, from nothing
        tables("tables-prompts", 128, 0, 128, 1.0, grow=1.0, end=0.0, cut=0.0, chunk=2048),
        # one new token of each of 64 sequences: rotated and appended
        rope("rope-step", "append", 64, base, "bf16", 128, "half", 2048),
        # chunks of long histories, scaled frequencies, odd token count
        rope("rope-chunks", "append", 8191, gqa7, "bf16", 128, "half", 1 << 18),
        # the prompts of the ordinary serving batch, half of each head, interleaved pairs
        rope("rope-prompts", "dense", 65536, base, "bf16", 64, "interleaved", 1024),
        # gradients of a small model in fp32, an odd share of the head
        rope("rope-gradient-f32", "gradient", 4100, tiny, "f32", 20, "half", 4096),
        # a single user's draft of five tokens to verify, where latency counts
        chunk("chunk-draft", 1, small, "bf16", (2000, 2000), (5, 5), 0.0, False),
        # the serving batch, one new token each
        chunk("chunk-singles", 64, base, "bf16", (700, 1044), (1, 1), 1.0, False),
        # single tokens beside pieces of prompts, odd group size
        chunk("chunk-mixed", 48, gqa7, "bf16", (0, 3000), (130, 700), 0.7, True),
        # a prompt in fp32 (the debugging workload) in two pieces
        chunk("chunk-f32", 2, tiny, "f32", (100, 150), (90, 156), 0.0, True),
        # long histories that grow by a thousand rows
        chunk("chunk-long", 8, base, "bf16", (16000, 31000), (1024, 1024), 0.0, False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("page_tables", "rope", "rope", "chunk_attn", "chunk_attn", "chunk_attn"))
    if op == "page_tables":
        n_seq = _log_int(rng, 1, 1024)
        chunk = _log_int(rng, 1, 2048)
        len_hi = rng.choice((0, _log_int(rng, 1, 8192)))
        grow, end, cut = rng.random() if len_hi else 1.0, 0.2 * rng.random(), 0.4 * rng.random()
        while n_seq > 1 and n_seq * chunk * grow > 140000:
            n_seq //= 2
        per_seq = -(-(len_hi + chunk) // PAGE) + rng.randint(0, 7)
        return dict(op=op, n_seq=n_seq, len_hi=len_hi, per_seq=per_seq, free=rng.choice((1.0, 1.0, 0.8)), grow=grow, end=end,
                    cut=cut, chunk=chunk)
    hq, hkv, d = rng.choice(HEADS)
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    if op == "rope":
        most = 65536 * 40 * 128 // ((hq + 2 * hkv) * d * (2 if dtype == "f32" else 1))
        rot = rng.choice((d, d, d // 2, 2 * rng.randint(1, d // 2)))
        return dict(op=op, form=rng.choice(("append", "append", "dense", "gradient")), tokens=_log_int(rng, 1, min(most, 131072)),
                    hq=hq, hkv=hkv, d=d, dtype=dtype, rot=rot, layout=rng.choice(("half", "half", "interleaved")),
                    far=_log_int(rng, 64, 1 << 20))
    batch = _log_int(rng, 1, 128)
    old_hi = rng.choice((0, _log_int(rng, 1, 32000), _log_int(rng, 1, 32000)))
    old_lo = old_hi if rng.random() < 0.3 else rng.randint(0, old_hi)
    new_hi = rng.choice((1, rng.randint(2, 16), _log_int(rng, 1, 4096)))
    new_lo = new_hi if rng.random() < 0.3 else rng.randint(1, new_hi)
    singles = 0.0 if rng.random() < 0.5 else rng.random()
    case = dict(op=op, batch=batch, hq=hq, hkv=hkv, d=d, dtype=dtype, old_lo=old_lo, old_hi=old_hi, new_lo=new_lo, new_hi=new_hi,
                singles=singles, lse=rng.random() < 0.5)
    # rows of the cache (with the plain form's 32-bit copies of them in mind) and products, as in the largest listed case
    rows = lambda: case["batch"] * (case["old_hi"] + case["new_hi"]) * hkv * d * (2 if dtype == "f32" else 1)        # noqa: E731
    pairs = lambda: case["batch"] * (case["old_hi"] + case["new_hi"]) * case["new_hi"] * hq * d * (12 if dtype == "f32" else 1)  # noqa: E731
    while case["batch"] > 1 and (rows() > 8 * 24000 * 8 * 128 or pairs() > 8 * 24000 * 1024 * 32 * 128):
        case["batch"] //= 2
    while case["new_hi"] > 1 and pairs() > 8 * 24000 * 1024 * 32 * 128:
        case["new_hi"] //= 2
        case["new_lo"] = min(case["new_lo"], case["new_hi"])
    while case["old_hi"] > 1 and rows() > 8 * 24000 * 8 * 128:
        case["old_hi"] //= 2
        case["old_lo"] = min(case["old_lo"], case["old_hi"])
    return case


def _spread(lo, hi, n, turn=0.6180339887498949):
    """n whole numbers over [lo, hi], the same for every seed, the largest among them."""
    return [hi - int((hi - lo + 1) * ((i * turn) % 1.0)) if hi > lo else hi for i in range(n)]


def _chunk_lens(case):
    """Rows held and rows added per sequence."""
    n = case["batch"]
    old, new = _spread(case["old_lo"], case["old_hi"], n), _spread(case["new_lo"], case["new_hi"], n, 0.4142135623730951)
    one = int(round(case["singles"] * n))
    return old, [1 if (i * 7919) % n < one else new[i] for i in range(n)]


def _table_lens(case):
    """Rows held and target lengths per sequence: `end` of them end, `cut` of them lose a few rows, `grow` of the others get a
    chunk and the rest one token."""
    n = case["n_seq"]
    held = _spread(case["len_hi"] // 2, case["len_hi"], n)
    target = []
    for i, h in enumerate(held):
        u, v = (i * 0.7548776662466927 + 0.31) % 1.0, (i * 0.5698402909980532 + 0.17) % 1.0
        if u < case["end"]:
            target.append(0)
        elif u < case["end"] + case["cut"]:
            target.append(max(0, h - 1 - i % 40))
        elif v < case["grow"]:
            target.append(h + max(1, case["chunk"] // 16 + int((case["chunk"] - case["chunk"] // 16) * ((i * 0.8191725133961645) % 1.0))))
        else:
            target.append(h + 1)
    return held, target


def _up(n):
    return -(-n // PAGE)


# ---------------------------------------------------------------------------------------------------- inputs
def _frequencies(case):
    """Radians per position of every pair, and the amplitude: from 10000, or, for far positions, from 500000 with the slow
    pairs' positions compressed eightfold, the fast ones kept, and a ramp between them."""
    half = case["rot"] // 2
    if case["far"] <= 8192:
        return [10000.0 ** (-i / half) for i in range(half)], 1.0
    out, factor, first = [], 8.0, 32768.0
    for i in range(half):
        f = 500000.0 ** (-i / half)
        turns = first * f / (2.0 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
        out.append(f * (keep + (1.0 - keep) / factor))
    return out, 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 23)
    kw = dict(generator=g, device="cuda")
    st = {"case": dict(case)}
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["op"] == "page_tables":
        held, target = _table_lens(case)
        n, per_seq = case["n_seq"], case["per_seq"]
        used = sum(_up(h) for h in held)
        taken = sum(max(0, _up(t) - _up(h)) for h, t in zip(held, target))
        back = sum(max(0, _up(h) - _up(t)) for h, t in zip(held, target))
        n_free = max(0, int(taken * case["free"]) - back) + (3 if case["free"] == 1.0 else 0)
        n_pages = used + n_free + 8
        perm = torch.randperm(n_pages, **kw).to(torch.int32)
        p = torch.arange(per_seq, device="cuda")
        have = torch.tensor([_up(h) for h in held], device="cuda")
        off = have.cumsum(0) - have
        mine = p[None, :] < have[:, None]
        table = torch.where(mine, perm[(off[:, None] + p[None, :]).clamp(max=n_pages - 1)], -1).to(torch.int32)
        free = torch.full((n_pages,), -1, **i32)
        free[:n_free] = perm[used:used + n_free]
        tokens = sum(max(0, t - h) for h, t in zip(held, target))
        st.update(held=torch.tensor(held, **i32), target=torch.tensor(target, **i32), table=table, free=free,
                  n_free=torch.tensor([n_free], **i32), n_pages=n_pages, tokens=_up(max(tokens, 1)) * PAGE)
        for name, size in (("held_out", n), ("n_free_out", 1), ("seq_len", n), ("cu_new", n + 1), ("positions", st["tokens"]),
                           ("slots", st["tokens"]), ("n_refused", 1)):
            st[name] = torch.zeros(size, **i32)
    elif case["op"] == "rope":
        t, hq, hkv, d, dt = case["tokens"], case["hq"], case["hkv"], case["d"], DTYPES[case["dtype"]]
        freq, st["amplitude"] = _frequencies(case)
        st["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        st["positions"] = torch.randint(0, case["far"], (t,), **kw).to(torch.int32)
        if case["form"] == "append":
            # the projection's output holds Q, K and V of a token side by side
            qkv = torch.randn(t, hq + 2 * hkv, d, **kw).to(dt)
            st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
            n_pages = _up(t) + min(t, 64)
            st["slots"] = torch.randperm(n_pages * PAGE, **kw)[:t].to(torch.int32)
            if t > 256:   # (a chunk's tokens fill pages one after the other)
                st["slots"] = (torch.randperm(n_pages, **kw)[:_up(t), None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)[:t].to(torch.int32)
            st["k_pages"] = torch.randn(n_pages, PAGE, hkv, d, **kw).to(dt)
            st["v_pages"] = torch.randn(n_pages, PAGE, hkv, d, **kw).to(dt)
            st["q_out"] = torch.zeros(t, hq, d, dtype=dt, device="cuda")
        else:
            st["q"], st["k"] = torch.randn(t, hq, d, **kw).to(dt), torch.randn(t, hkv, d, **kw).to(dt)
            st["q_out"], st["k_out"] = torch.zeros_like(st["q"]), torch.zeros_like(st["k"])
    else:
        b, hq, hkv, d, dt = case["batch"], case["hq"], case["hkv"], case["d"], DTYPES[case["dtype"]]
        old, new = _chunk_lens(case)
        lens = [x + y for x, y in zip(old, new)]
        st["lens"], st["new"] = lens, new
        per_seq = _up(max(lens)) + b % 3
        n_pages = b * per_seq
        st["table"] = torch.randperm(n_pages, **kw).to(torch.int32).reshape(b, per_seq)
        st["k_pages"] = torch.randn(n_pages, PAGE, hkv, d, **kw).to(dt)
        st["v_pages"] = torch.randn(n_pages, PAGE, hkv, d, **kw).to(dt)
        cu = [0]
        for x in new:
            cu.append(cu[-1] + x)
        st["cu"], st["cu_new"], st["seq_len"] = cu, torch.tensor(cu, **i32), torch.tensor(lens, **i32)
        # queries that look at some keys more than at others, as trained ones do
        st["q"] = (1.5 * torch.randn(cu[-1], hq, d, **kw)).to(dt)
        st["o"] = torch.zeros_like(st["q"])
        if case["lse"]:
            st["lse"] = torch.zeros(hq, cu[-1], device="cuda")
    if own:
        st["handles"] = _handles(st)
    return st


# ---------------------------------------------------------------------------------------------------- plain forms
def _plain_page_tables(st):
    c = st["case"]
    cap, n_tok, n_pages = c["per_seq"] * PAGE, st["tokens"], st["n_pages"]
    h, t = st["held"].long().clamp(0, cap), st["target"].long().clamp(min=0)
    new = (t - h).clamp(min=0)
    end = new.cumsum(0)
    fits = (new == 0) | ((t <= cap) & (end <= n_tok))
    have, want = (h + PAGE - 1) // PAGE, (t + PAGE - 1) // PAGE
    need = torch.where(fits, (want - have).clamp(min=0), 0)
    back = (have - want).clamp(min=0)
    back_at = st["n_free"].long() + back.cumsum(0) - back
    room = (st["n_free"].long() + back.sum()).clamp(max=n_pages)
    need_end = need.cumsum(0)
    granted = fits & ((need == 0) | (need_end <= room))
    # pages given back go on top of the list of free ones, in order
    p = torch.arange(c["per_seq"], device="cuda")[None, :]
    leaving = (p >= want[:, None]) & (p < have[:, None])
    at = torch.where(leaving, back_at[:, None] + p - want[:, None], n_pages).clamp(max=n_pages)
    stack = torch.cat((st["free"], st["free"][:1]))
    stack[at] = torch.where(leaving, st["table"], stack[at])
    # and pages are taken from its top
    coming = granted[:, None] & (p >= have[:, None]) & (p < want[:, None])
    take = torch.where(coming, room - 1 - (need_end - need)[:, None] - (p - have[:, None]), 0)
    table = torch.where(coming, stack[take], st["table"])
    st["free"].copy_(stack[:n_pages])
    st["table"].copy_(table)
    st["held_out"].copy_(torch.where(granted, t, h))
    st["n_free_out"].copy_(room - torch.where(granted, need, 0).sum())
    st["seq_len"].copy_(torch.where(granted, t, 0))
    st["cu_new"][1:] = end.clamp(max=n_tok)
    st["n_refused"].copy_((~granted).sum())
    j = torch.arange(n_tok, device="cuda")
    b = torch.searchsorted(end, j, right=True)
    live = b < c["n_seq"]
    b = b.clamp(max=c["n_seq"] - 1)
    live = live & granted[b]
    pos = h[b] + j - (end - new)[b]
    row = torch.where(live, pos, 0)
    st["positions"].copy_(torch.where(live, pos, -1))
    st["slots"].copy_(torch.where(live, table[b, row // PAGE].long() * PAGE + row % PAGE, -1))
    return _table_outputs(st)


def _table_outputs(st):
    return {name: st[name] for name in ("table", "free", "held_out", "n_free_out", "seq_len", "cu_new", "positions", "slots", "n_refused")}


def _turned(x, st, dtype):
    """The rows of x [T, H, D] turned by their positions (back, for a gradient), in `dtype`."""
    c = st["case"]
    rot, half = c["rot"], c["rot"] // 2
    angle = st["positions"].double()[:, None] * st["freq"][None, :]
    cos, sin = (torch.cos(angle) * st["amplitude"]).to(dtype)[:, None], (torch.sin(angle) * st["amplitude"]).to(dtype)[:, None]
    if c["form"] == "gradient":
        sin = -sin
    y = x.to(dtype, copy=True)
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if c["layout"] == "interleaved" else (slice(0, half), slice(half, rot))
    a, b = y[..., first], y[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, a * sin + b * cos
    return y


def _plain_rope(st):
    c = st["case"]
    st["q_out"].copy_(_turned(st["q"], st, torch.float32))
    if c["form"] != "append":
        st["k_out"].copy_(_turned(st["k"], st, torch.float32))
        return {"q": st["q_out"], "k": st["k_out"]}
    at = st["slots"].long()
    st["k_pages"].view(-1, c["hkv"], c["d"])[at] = _turned(st["k"], st, torch.float32).to(st["k_pages"].dtype)
    st["v_pages"].view(-1, c["hkv"], c["d"])[at] = st["v"]
    return {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}


def _plain_chunk_attn(st):
    c = st["case"]
    hkv, grp, d = c["hkv"], c["hq"] // c["hkv"], c["d"]
    for i, (n, m) in enumerate(zip(st["lens"], st["new"])):
        page = st["table"][i, :_up(n)].long()
        k = st["k_pages"][page].flatten(0, 1)[:n].float().permute(1, 2, 0)                        # [Hkv, D, n]
        v = st["v_pages"][page].flatten(0, 1)[:n].float().permute(1, 0, 2)                        # [Hkv, n, D]
        for a in range(0, m, 512):
            e = min(m, a + 512)
            lo, hi = st["cu"][i] + a, st["cu"][i] + e
            q = st["q"][lo:hi].float().reshape(e - a, hkv, grp, d).permute(1, 2, 0, 3).reshape(hkv, grp * (e - a), d)
            s = torch.matmul(q, k).reshape(hkv, grp, e - a, n) * (1.0 / math.sqrt(d))
            hidden = torch.arange(n, device="cuda")[None, :] > (n - m + torch.arange(a, e, device="cuda"))[:, None]
            s = s.masked_fill_(hidden, float("-inf"))
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul((p / total).reshape(hkv, grp * (e - a), n), v).reshape(hkv, grp, e - a, d)
            st["o"][lo:hi] = o.permute(2, 0, 1, 3).reshape(e - a, c["hq"], d).to(st["o"].dtype)
            if c["lse"]:
                st["lse"][:, lo:hi] = (top + torch.log(total)).reshape(c["hq"], e - a)
    return {"o": st["o"], "lse": st["lse"]} if c["lse"] else {"o": st["o"]}


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _handles(st):
    """What a program keeps beside its tensors: descriptions of the model, the cache, the pool and the step, the workspace."""
    from paper_2507_00715_b200 import binding as B

    c = st["case"]
    h = {"B": B}
    if c["op"] == "page_tables":
        h["pool"] = B.make_page_pool(st["table"], st["held"], st["free"], st["n_free"])
        h["step"] = B.make_step(st["cu_new"], st["seq_len"], st["positions"], st["slots"], st["n_refused"])
        need = B.earn_page_tables_workspace_bytes(c["n_seq"])
    else:
        h["model"] = B.make_model(1, 1, c["hq"], c["hkv"], c["d"], c["dtype"])
        need = 0
    if c["op"] == "rope":
        h["rope"] = B.make_rope(st["freq"], interleaved=c["layout"] == "interleaved", amplitude=st["amplitude"])
        if c["form"] == "append":
            h["cache"] = B.make_paged_cache(st["k_pages"], st["v_pages"], pages_per_seq=st["k_pages"].shape[0])
    elif c["op"] == "chunk_attn":
        h["cache"] = B.make_paged_cache(st["k_pages"], st["v_pages"], st["table"], st["seq_len"], max_len=max(st["lens"]))
        need = B.earn_paged_chunk_workspace_bytes(h["model"], c["batch"], st["cu"][-1], h["cache"])
    if need:
        h["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        B.earn_workspace_init(h["workspace"])
    return h


def _own_call(st):
    if "handles" not in st:
        st["handles"] = _handles(st)
    h, c = st["handles"], st["case"]
    B = h["B"]
    if c["op"] == "page_tables":
        B.earn_page_tables(c["n_seq"], st["target"], h["pool"], h["step"], st["held_out"], st["n_free_out"], h["workspace"])
        return _table_outputs(st)
    if c["op"] == "chunk_attn":
        B.earn_paged_chunk_attn(h["model"], c["batch"], 0, st["cu"][-1], st["cu_new"], st["q"], h["cache"], st["o"], st.get("lse"),
                                h["workspace"])
        return {"o": st["o"], "lse": st["lse"]} if c["lse"] else {"o": st["o"]}
    if c["form"] == "append":
        B.earn_rope_append(h["model"], 0, h["rope"], c["tokens"], st["positions"], st["slots"], st["q"], st["k"], st["v"], st["q_out"],
                           h["cache"])
        return {"q": st["q_out"], "k_pages": st["k_pages"], "v_pages": st["v_pages"]}
    B.earn_rope(h["model"], h["rope"], c["tokens"], st["positions"], st["q"], st["k"], st["q_out"], st["k_out"],
                inverse=c["form"] == "gradient")
    return {"q": st["q_out"], "k": st["k_out"]}


def run(state):
    if own:
        return _own_call(state)
    return {"page_tables": _plain_page_tables, "rope": _plain_rope, "chunk_attn": _plain_chunk_attn}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------- necessary work
def work(case):
    if case["op"] == "page_tables":
        held, target = _table_lens(case)
        tokens = sum(max(0, t - h) for h, t in zip(held, target))
        moved = sum(abs(_up(t) - _up(h)) for h, t in zip(held, target))
        return {"bytes": 20 * case["n_seq"] + 8 * tokens + 8 * moved, "flops": 0}
    e = 4 if case["dtype"] == "f32" else 2
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "rope":
        heads = hq + (2 if case["form"] == "append" else 1) * hkv
        return {"bytes": case["tokens"] * (2 * heads * d * e + (8 if case["form"] == "append" else 4)),
                "flops": case["tokens"] * (hq + hkv) * case["rot"] * 3}
    old, new = _chunk_lens(case)
    seen = sum(m * x + m * (m + 1) // 2 for x, m in zip(old, new))
    rows, tokens = sum(old) + sum(new), sum(new)
    return {"bytes": rows * 2 * hkv * d * e + tokens * hq * (2 * d * e + (4 if case["lse"] else 0)), "flops": 4 * hq * d * seen}


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """The rotations and the attention by their definitions in 64 bits.  The page tables are whole numbers."""
    if case["op"] == "page_tables":
        return None
    st = prepare(case, seed)
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    if case["op"] == "rope":
        rot, half = case["rot"], case["rot"] // 2
        way = -1.0 if case["form"] == "gradient" else 1.0
        turn = torch.polar(torch.full((case["tokens"], half), st["amplitude"], dtype=torch.float64, device="cuda"),
                           way * st["positions"].double()[:, None] * st["freq"])

        def turned(x):
            y = x.double()
            pairs = y[..., :rot].unflatten(-1, (half, 2) if case["layout"] == "interleaved" else (2, half))
            if case["layout"] != "interleaved":
                pairs = pairs.transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
            if case["layout"] != "interleaved":
                z = z.transpose(-1, -2)
            return torch.cat((z.flatten(-2), y[..., rot:]), -1)

        if case["form"] != "append":
            return {"q": turned(st["q"]), "k": turned(st["k"])}
        pages = st["k_pages"].double()
        pages.view(-1, hkv, d)[st["slots"].long()] = turned(st["k"])
        return {"q": turned(st["q"]), "k_pages": pages, "v_pages": None}
    o = torch.zeros(st["cu"][-1], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(hq, st["cu"][-1], dtype=torch.float64, device="cuda")
    for i, (n, m) in enumerate(zip(st["lens"], st["new"])):
        page = st["table"][i].long()
        key, val = (st[x][page].flatten(0, 1)[:n] for x in ("k_pages", "v_pages"))
        for a in range(0, m, 1024):
            e = min(m, a + 1024)
            lo, seen = st["cu"][i] + a, n - m + e
            later = torch.arange(seen, device="cuda")[None, :] > torch.arange(n - m + a, seen, device="cuda")[:, None]
            for x in range(hq):
                logit = (st["q"][lo:lo + e - a, x].double() / math.sqrt(d)) @ key[:seen, x * hkv // hq].double().T
                logit[later] = -math.inf
                lse[x, lo:lo + e - a] = torch.logsumexp(logit, -1)
                o[lo:lo + e - a, x] = torch.softmax(logit, -1) @ val[:seen, x * hkv // hq].double()
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}
