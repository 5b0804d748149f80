"""Call sequencing for one batch: owns the caches and workspace and issues the C-ABI calls in the
order of the hot path (Section 3.2, "Inference").  No arithmetic happens here."""
from __future__ import annotations

from typing import List, Optional

import numpy as np
import torch

from . import binding as B


class EarnSession:
    """One batch of prompts through prefill and decode.

    Layers ``l < split_k`` keep a reference to the caller's packed K/V (read in place during decode);
    layers ``l >= split_k`` own a paged compact register cache.  Every layer owns a private
    (generated-token) cache of ``max_new`` tokens per beam.
    """

    def __init__(self, n_layers: int, split_k: int, n_q_heads: int, n_kv_heads: int, head_dim: int, dtype: torch.dtype,
                 cu_seqlens: np.ndarray, r_head: int, r_tail: int, beams: int = 1, max_new: int = 1,
                 softmax_scale: float = 0.0, device="cuda", paged_shuffle_seed: Optional[int] = None,
                 paged_private_seed: Optional[int] = None):
        self.device = torch.device(device)
        self.dtype = dtype
        self.model = B.make_model(n_layers, split_k, n_q_heads, n_kv_heads, head_dim, dtype, softmax_scale)
        self.batch = B.Batch(cu_seqlens, r_head, r_tail, device=self.device)
        self.beams, self.max_new = beams, max(1, max_new)
        self.n_layers, self.split_k = n_layers, split_k
        self.Hq, self.Hkv, self.D = n_q_heads, n_kv_heads, head_dim
        nb, R = self.batch.batch, r_head + r_tail
        self.R = R
        self.pages_per_seq = max(1, -(-R // B.PAGE_TOKENS))
        self.n_pages = max(1, nb * self.pages_per_seq)
        # an optional scattered page table exercises the paged addressing; None = identity layout
        self.block_table = None
        if paged_shuffle_seed is not None:
            perm = np.random.Generator(np.random.Philox(paged_shuffle_seed)).permutation(self.n_pages)
            self.block_table = torch.from_numpy(perm.astype(np.int32).reshape(nb, self.pages_per_seq)).to(self.device)
        kw = dict(device=self.device, dtype=dtype)
        self.k_shared: List[Optional[torch.Tensor]] = [None] * n_layers
        self.v_shared: List[Optional[torch.Tensor]] = [None] * n_layers
        self.k_full: List[Optional[torch.Tensor]] = [None] * n_layers
        self.v_full: List[Optional[torch.Tensor]] = [None] * n_layers
        self.released = set()   # full layers whose packed K/V another cache has taken over
        self.k_priv, self.v_priv = [], []
        # the private (generated-token) segment: flat slabs, or pages behind a scattered table (one table for all layers)
        self.priv_table, self.priv_pages_per_beam, self.n_priv_pages = None, 0, 0
        if paged_private_seed is not None:
            self.priv_pages_per_beam = -(-self.max_new // B.PAGE_TOKENS)
            self.n_priv_pages = max(1, nb * beams * self.priv_pages_per_beam)
            perm = np.random.Generator(np.random.Philox(paged_private_seed)).permutation(self.n_priv_pages)
            self.priv_table = torch.from_numpy(perm.astype(np.int32).reshape(nb * beams, self.priv_pages_per_beam)).to(self.device)
        for layer in range(n_layers):
            if layer >= split_k:
                self.k_shared[layer] = torch.zeros(self.n_pages, B.PAGE_TOKENS, n_kv_heads, head_dim, **kw)
                self.v_shared[layer] = torch.zeros(self.n_pages, B.PAGE_TOKENS, n_kv_heads, head_dim, **kw)
            if self.priv_table is not None:
                self.k_priv.append(torch.zeros(self.n_priv_pages, B.PAGE_TOKENS, n_kv_heads, head_dim, **kw))
                self.v_priv.append(torch.zeros(self.n_priv_pages, B.PAGE_TOKENS, n_kv_heads, head_dim, **kw))
            else:
                self.k_priv.append(torch.zeros(nb * beams, self.max_new, n_kv_heads, head_dim, **kw))
                self.v_priv.append(torch.zeros(nb * beams, self.max_new, n_kv_heads, head_dim, **kw))
        self.reg_idx = torch.zeros(nb, max(R, 1), dtype=torch.int32, device=self.device)
        self.lineage = [torch.zeros(nb * beams, self.max_new, dtype=torch.int32, device=self.device) for _ in range(2)]
        self.lineage_cur: Optional[int] = None      # None = identity table
        ws_bytes = B.earn_workspace_bytes(self.model, self.batch, beams)
        self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=self.device)
        B.earn_workspace_init(self.workspace)

    # ---- cache descriptors
    def cache(self, layer: int) -> B.EarnCache:
        lin = None if self.lineage_cur is None else self.lineage[self.lineage_cur]
        return B.make_cache(self.k_shared[layer], self.v_shared[layer], self.block_table, self.pages_per_seq,
                            self.n_pages, self.k_priv[layer], self.v_priv[layer], lin, self.beams, self.max_new,
                            self.reg_idx, self.priv_table, self.priv_pages_per_beam, self.n_priv_pages)

    # ---- prefill
    def release_prompt(self, layer: int) -> None:
        """Lets go of the packed K/V of a layer < k that ``prefill_layer`` was given (a BudgetedLayers holds its rows from then
        on).  decode_layer refuses the layer until it is prefilled again."""
        if not 0 <= layer < self.split_k:
            raise ValueError(f"layer {layer} is not a full layer")
        for kv in (self.k_full, self.v_full):
            if kv[layer] is not None and kv[layer].is_cuda:
                kv[layer].record_stream(torch.cuda.current_stream(kv[layer].device))   # (what is enqueued here still reads it)
            kv[layer] = None
        self.released.add(layer)

    def prefill_layer(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                      out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                      q_reg: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Layer < k: full causal attention, returns O [total,Hq,D] and keeps k, v for decode.
        Layer >= k: compaction then register attention, returns O' [B,R,Hq,D]."""
        if layer < self.split_k:
            o = out if out is not None else torch.empty_like(q)
            B.earn_prefill_attn(self.model, self.batch, layer, q, k, v, o, lse, self.workspace)
            self.k_full[layer], self.v_full[layer] = k, v
            self.released.discard(layer)
            return o
        nb = self.batch.batch
        if q_reg is None:
            q_reg = torch.empty(nb, self.R, self.Hq, self.D, device=self.device, dtype=self.dtype)
        o = out if out is not None else torch.empty_like(q_reg)
        cache = self.cache(layer)
        B.earn_compact_kv(self.model, self.batch, layer, k, v, cache, q, q_reg)
        B.earn_register_attn(self.model, self.batch, layer, q_reg, cache, o, self.workspace)
        self.last_q_reg = q_reg
        return o

    def register_layer_fused(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                             out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Layer >= k in one launch: compaction and register attention together (no gathered copy of the queries).
        Returns O' [B,R,Hq,D]; the compact cache and reg_idx are left as prefill_layer leaves them."""
        o = out if out is not None else torch.empty(self.batch.batch, self.R, self.Hq, self.D, device=self.device,
                                                    dtype=self.dtype)
        B.earn_compact_register_attn(self.model, self.batch, layer, q, k, v, self.cache(layer), o, self.workspace)
        return o

    def set_projection(self, d_model: int, max_pos: int, theta: float = 10000.0, rms_eps: float = 1e-6) -> None:
        """Rotary tables (angles pos * theta^(-2i/D), evaluated in double, stored fp32) and the scratch the
        hidden-state form of the register layers needs."""
        inv = theta ** (-torch.arange(0, self.D, 2, dtype=torch.float64) / self.D)
        ang = torch.arange(max_pos, dtype=torch.float64)[:, None] * inv[None, :]
        self.rope_cos = torch.cos(ang).float().to(self.device)
        self.rope_sin = torch.sin(ang).float().to(self.device)
        self.d_model, self.rms_eps = d_model, rms_eps
        self.x_norm = torch.empty(max(self.batch.batch * self.R, 1), d_model, device=self.device, dtype=self.dtype)

    def register_layer_from_hidden(self, layer: int, x: torch.Tensor, w_norm: torch.Tensor, w_qkv: torch.Tensor,
                                   x_is_compact: bool = False, out: Optional[torch.Tensor] = None,
                                   q_reg: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Layer >= k from the hidden states: projection of the register rows into the compact cache, then register
        attention.  Returns O' [B,R,Hq,D]; call set_projection() first."""
        nb = self.batch.batch
        if q_reg is None:
            q_reg = torch.empty(nb, self.R, self.Hq, self.D, device=self.device, dtype=self.dtype)
        o = out if out is not None else torch.empty_like(q_reg)
        cache = self.cache(layer)
        proj = B.make_proj(self.d_model, self.rope_cos, self.rope_sin, self.rms_eps, x_is_compact)
        B.earn_register_qkv(self.model, self.batch, layer, proj, x, w_norm, w_qkv, self.x_norm, cache, q_reg,
                            self.workspace)
        B.earn_register_attn(self.model, self.batch, layer, q_reg, cache, o, self.workspace)
        self.last_q_reg = q_reg
        return o

    # ---- decode
    def begin_step(self, step: int, parents: Optional[torch.Tensor]) -> None:
        """Re-parent the beams before decode step `step` (>= 2); parents: int32 device [B*W]."""
        if parents is None or self.beams == 1 or step < 2:
            return
        nxt = 0 if self.lineage_cur != 0 else 1
        lin_in = None if self.lineage_cur is None else self.lineage[self.lineage_cur]
        B.earn_beam_reparent(self.batch.batch, self.beams, self.max_new, step, parents, lin_in, self.lineage[nxt])
        self.lineage_cur = nxt

    def decode_layer(self, layer: int, step: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
        if layer in self.released:
            raise ValueError(f"layer {layer}: the prompt's keys and values were released")
        o = out if out is not None else torch.empty_like(q)
        B.earn_decode_attn(self.model, self.batch, layer, step, q, k_new, v_new, self.cache(layer), o,
                           self.k_full[layer], self.v_full[layer], self.workspace)
        return o

    def device_status(self) -> int:
        return B.earn_device_status(self.workspace)

    # ---- accounting (Eq. 9 on the actual buffers): KV entries per kv head held after `generated` steps (a released layer's
    # rows are in another cache, which counts them)
    def kv_entries(self, generated: int) -> int:
        lens = np.diff(self.batch.cu_host)
        total = 0
        for layer in range(self.n_layers):
            if layer in self.released:
                continue
            shared = int(lens.sum()) if layer < self.split_k else self.R * len(lens)
            total += shared + len(lens) * self.beams * generated
        return total


class BudgetedLayers:
    """The full layers (``l < split_k``) of a session's batch with at most ``budget`` rows per sequence and kv head.

    After the prefill of a layer (with its softmax denominators) ``take_prompt`` weighs the prompt's rows by the last
    ``n_obs`` queries and copies the budget's worth into pages of its own.  The session keeps the packed K/V that its prefill
    was given all the same, unless ``take_prompt`` is told to ``release`` them (its own decode of the layer needs them).  A decode
    step is ``begin_step``, ``decode_layer`` for every full layer (the register layers stay with the session), and
    ``end_step``.  While the rows stay below the budget there is room for the session's ``max_new`` tokens, as in its own
    cache (``begin_step`` counts them on the host, so a captured step is replayed at the budget only); at the budget there is no
    end.  By default the suffix registers (at least one row) do the weighing.  One beam per sequence.

    The policy's last tokens are the newest ones, generated ones included, so it lets go of the suffix registers as the
    sequence grows.  They stay all the same: those among the prompt's last ``n_last`` rows (all of them by default) enter
    the cache with a weight of +inf, which no step changes.  ``n_first`` is the number of prefix registers by default;
    ``n_last`` that of suffix registers, or as many as the budget holds beside the registers.  A budget that the
    sequences reach and that is too small for the first rows, the suffix registers and the last rows together is refused.
    """

    def __init__(self, session: EarnSession, budget: int, n_first: Optional[int] = None, n_last: Optional[int] = None,
                 n_obs: Optional[int] = None, paged_shuffle_seed: Optional[int] = None):
        if session.beams != 1:
            raise ValueError("a budgeted cache holds one beam per sequence")
        self.session, self.budget = session, budget
        batch, dev = session.batch, session.device
        r_head, r_tail = batch.c.n_head_reg, batch.c.n_tail_reg
        n_first = r_head if n_first is None else n_first
        pinned = r_tail if n_last is None else min(r_tail, max(n_last, 0))   # suffix registers that stay for good
        if n_last is None:
            n_last = max(0, min(r_tail, budget - n_first - pinned))
        self.policy = B.make_evict(budget, n_first, n_last)
        self.n_obs = max(1, r_tail) if n_obs is None else n_obs
        nb = batch.batch
        lens = np.diff(batch.cu_host)
        self.pinned_rows = torch.from_numpy((batch.cu_host[1:, None] - np.arange(1, pinned + 1)).reshape(-1).astype(np.int64)).to(dev)
        longest = int(lens.max()) if nb else 0
        held = max(1, min(longest + session.max_new, budget + 1))   # rows during a step
        self.steps_left = session.max_new if held <= budget else None
        if held > budget and n_first + pinned + n_last > budget:
            raise ValueError(f"a budget of {budget} rows does not hold {n_first} first rows, {pinned} suffix registers and "
                             f"{n_last} last rows")
        self.pages_per_seq = max(1, -(-held // B.PAGE_TOKENS))
        n_pages = max(1, nb * self.pages_per_seq)
        self.block_table = None
        if paged_shuffle_seed is not None:
            perm = np.random.Generator(np.random.Philox(paged_shuffle_seed)).permutation(n_pages)
            self.block_table = torch.from_numpy(perm.astype(np.int32).reshape(nb, self.pages_per_seq)).to(dev)
        shape, rows = (n_pages, B.PAGE_TOKENS, session.Hkv, session.D), (nb, session.Hkv, B.PAGE_TOKENS * self.pages_per_seq)
        full = range(session.split_k)
        self.k_pages = [torch.zeros(shape, device=dev, dtype=session.dtype) for _ in full]
        self.v_pages = [torch.zeros(shape, device=dev, dtype=session.dtype) for _ in full]
        self.weight = [torch.zeros(rows, device=dev, dtype=torch.float32) for _ in full]
        self.pos = [torch.zeros(rows, device=dev, dtype=torch.int32) for _ in full]
        self.seq_len = torch.from_numpy(np.minimum(lens, budget).astype(np.int32)).to(dev)
        self.new_pos = torch.from_numpy((lens - 1).astype(np.int32)).to(dev)
        self.prompt_weight = torch.empty(session.Hkv, max(batch.c.total_tokens, 1), device=dev, dtype=torch.float32)
        self.caches = [B.make_paged_cache(self.k_pages[i], self.v_pages[i], self.block_table, self.seq_len, held, self.pages_per_seq)
                       for i in full]
        if self.caches:
            self.workspace = torch.empty(B.earn_paged_workspace_bytes(session.model, nb, self.caches[0]), dtype=torch.uint8, device=dev)
            B.earn_workspace_init(self.workspace)

    def take_prompt(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, lse: torch.Tensor,
                    release: bool = False) -> None:
        """q, k, v of a full layer (packed) and the lse its prefill wrote -> the layer's pages, weights and positions.
        release: the session lets go of the packed K/V, which are freed once the caller drops them too."""
        ses = self.session
        B.earn_key_weights(ses.model, ses.batch, layer, self.n_obs, q, k, lse, self.prompt_weight, ses.workspace)
        if self.pinned_rows.numel():
            self.prompt_weight.index_fill_(1, self.pinned_rows, float("inf"))
        B.earn_evict_prompt_kv(ses.model, ses.batch, layer, self.policy, k, v, self.prompt_weight, self.caches[layer],
                               self.weight[layer], self.pos[layer], self.workspace)
        if release:
            ses.release_prompt(layer)

    def begin_step(self) -> None:
        if self.steps_left is not None:
            if self.steps_left == 0:
                raise ValueError(f"a session of max_new = {self.session.max_new} has no room for another token")
            self.steps_left -= 1
        self.seq_len.add_(1)
        self.new_pos.add_(1)

    def decode_layer(self, layer: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The layer's decode step and its return to the budget; O [B, Hq, D]."""
        o = out if out is not None else torch.empty_like(q)
        nb, w, p = self.session.batch.batch, self.weight[layer], self.pos[layer]
        B.earn_paged_decode_attn(self.session.model, nb, layer, q, k_new, v_new, self.caches[layer], o, w, w, self.new_pos, p,
                                 self.workspace)
        B.earn_evict_kv(self.session.model, nb, layer, self.policy, self.caches[layer], w, p, w, p, self.workspace)
        return o

    def end_step(self) -> None:
        self.seq_len.clamp_(max=self.budget)

    def kv_entries(self, generated: int) -> int:
        """KV entries per kv head that the session and the budgeted layers hold after `generated` steps of the layers: the rows
        within the budget, the register layers' rows, and the packed prompts that were not released."""
        ses, lens = self.session, np.diff(self.session.batch.cu_host)
        total = 0
        for layer in range(ses.n_layers):
            if layer < ses.split_k:
                total += int(np.minimum(lens + generated, self.budget).sum()) + (0 if layer in ses.released else int(lens.sum()))
            else:
                total += (ses.R + generated) * len(lens)
        return total

    def device_status(self) -> int:
        """The first error in the status words of the session's workspace, into which the weighing of the prompt's rows reports
        (after one of those the rows kept may be the wrong ones), and of the workspace of the pages."""
        status = self.session.device_status()
        return status if status != B.EARN_OK or not self.caches else B.earn_device_status(self.workspace)
