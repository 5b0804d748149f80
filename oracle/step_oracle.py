"""Plain definitions, in 64 bits on the CPU, of a step of several new tokens over a paged cache: page tables, rotary positions,
causal attention of the new tokens over the paged lists.  Written from the definitions in ``include/earn.h``; loops where the
kernels scan."""
import math

import numpy as np

PAGE = 16


def page_tables(target, held, table, free, n_free, n_tokens):
    """Lists in, dict of arrays out (table and free are copied).  Mirrors the documented order: first every page given back,
    then the sequences one after the other, none overtaken."""
    n_seq, per_seq = table.shape
    table, stack = table.copy(), list(free[:n_free])
    up = lambda rows: -(-rows // PAGE)  # noqa: E731
    out = dict(held=np.array(held), seq_len=np.zeros(n_seq, int), cu=np.zeros(n_seq + 1, int), positions=np.full(n_tokens, -1),
               slots=np.full(n_tokens, -1), refused=0)
    for b in range(n_seq):
        for p in range(up(max(target[b], 0)), up(held[b])):
            stack.append(table[b, p])
    pushed = list(stack)
    first, short, need_so_far, room = 0, False, 0, len(stack)
    for b in range(n_seq):
        t, h = max(target[b], 0), held[b]
        grow = max(t - h, 0)
        out["cu"][b + 1] = min(first + grow, n_tokens)
        fits = grow == 0 or (first + grow <= n_tokens and t <= per_seq * PAGE)
        need = max(up(t) - up(h), 0) if fits else 0
        need_so_far += need
        short = short or need_so_far > room
        if not fits or (need > 0 and short):
            out["refused"] += 1
        else:
            for p in range(up(h), up(h) + need):
                table[b, p] = stack.pop()
            out["held"][b] = out["seq_len"][b] = t
            for i in range(grow):
                row = h + i
                out["positions"][first + i] = row
                out["slots"][first + i] = table[b, row // PAGE] * PAGE + row % PAGE
        first += grow
    return dict(out, table=table, stack=np.array(stack, int), pushed=np.array(pushed, int))


def rotate(x, positions, freq, interleaved=False, amplitude=1.0, inverse=False):
    """x [T, H, D] turned by its rows' positions."""
    y = x.astype(np.float64).copy()
    half = len(freq)
    sign = -1.0 if inverse else 1.0
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = positions.astype(np.float64) * freq[i]
        c, s = (amplitude * np.cos(angle))[:, None], (sign * amplitude * np.sin(angle))[:, None]
        xa, xb = x[:, :, a].astype(np.float64), x[:, :, b].astype(np.float64)
        y[:, :, a], y[:, :, b] = xa * c - xb * s, xa * s + xb * c
    return y


def chunk_attention(q, k_rows, v_rows, n_new, seq_len, scale=None):
    """q [sum n_new, Hq, D]; k_rows, v_rows: per sequence [>= seq_len, Hkv, D].  Returns o, lse [Hq, sum n_new], and the weighted
    mean of |v| (for bounds)."""
    total, hq, d = q.shape
    hkv = k_rows[0].shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o, mag, lse = np.zeros((total, hq, d)), np.zeros((total, hq, d)), np.full((hq, total), -np.inf)
    row = 0
    for b, n in enumerate(n_new):
        for i in range(n):
            seen = seq_len[b] - n + i + 1
            if seen > 0:
                for h in range(hq):
                    kv = h * hkv // hq
                    s = k_rows[b][:seen, kv].astype(np.float64) @ q[row, h].astype(np.float64) * scale
                    m = s.max()
                    if m > -np.inf:
                        p = np.exp(s - m)
                        lse[h, row] = m + np.log(p.sum())
                        p /= p.sum()
                        o[row, h] = p @ v_rows[b][:seen, kv].astype(np.float64)
                        mag[row, h] = p @ np.abs(v_rows[b][:seen, kv].astype(np.float64))
            row += 1
    return o, lse, mag
