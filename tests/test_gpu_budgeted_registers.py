"""The suffix registers of a session's budgeted layers: they are still held, and attended to, after more steps than the policy's
last tokens, when `n_last` has long moved on to generated tokens."""
import numpy as np
import pytest
import torch

from oracle import earn_oracle as orc
from paper_2507_00715_b200 import binding as B
from paper_2507_00715_b200 import workloads as wl
from paper_2507_00715_b200.session import BudgetedLayers
from parity_util import assert_close, make_session, to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("budget,n_last,kept,recent", [(24, None, 4, 4), (64, None, 4, 4), (10, None, 4, 2), (8, None, 4, 0), (16, 8, 4, 8),
                                                       (20, 2, 2, 2), (20, 0, 0, 0)])
def test_registers_stay(dtype, d, budget, n_last, kept, recent):
    """Twelve steps with four registers at either end: `kept` suffix registers and the `recent` newest tokens are held after
    every one of them, the outputs are the oracle's over the rows that `pos` names, and the others' weights stay finite."""
    w = wl.Workload("registers", batch=3, n_layers=2, split_k=2, n_q_heads=4, n_kv_heads=2, head_dim=d, dtype=dtype, prompt_len=0,
                    lens=(90, 40, 131), r_head=4, r_tail=4, decode_steps=12, seed=52)
    cu, lens = wl.cu_seqlens(w), [int(n) for n in wl.seqlens(w)]
    ses = make_session(w)
    bud = BudgetedLayers(ses, budget, n_last=n_last, paged_shuffle_seed=3)
    rows = []
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
            n_before = [min(n + step - 1, budget) for n in lens]
            q, k, v = wl.decode_qkv(w, layer, step, "cuda")
            o = bud.decode_layer(layer, q, k, v)
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
        for layer in range(2):
            p, weight = bud.pos[layer].cpu().numpy(), bud.weight[layer].cpu().numpy()
            for b, n in enumerate(lens):
                m = int(bud.seq_len[b])
                for h in range(2):
                    held = p[b, h, :m].tolist()
                    assert len(set(held)) == m and set(range(w.r_head)) <= set(held)
                    assert set(range(n - kept, n)) <= set(held), (step, layer, b, h)
                    assert set(range(n + step - recent, n + step)) <= set(held)
                    for at, x in zip(held, weight[b, h, :m]):
                        assert np.isposinf(x) if n - kept <= at < n else np.isfinite(x)
    assert bud.device_status() == B.EARN_OK


def test_a_wait_that_ran_out_in_the_sessions_workspace_is_reported():
    w = wl.Workload("status", batch=1, n_layers=1, split_k=1, n_q_heads=4, n_kv_heads=2, head_dim=64, dtype="bf16", prompt_len=0,
                    lens=(20,), r_head=2, r_tail=2, decode_steps=1, seed=1)
    ses = make_session(w)
    bud = BudgetedLayers(ses, 16)
    assert bud.device_status() == B.EARN_OK
    B.earn_selftest_wait_timeout(ses.workspace, 1000)      # a bounded wait on a barrier that nothing completes, in place of the kernel's
    assert bud.device_status() == B.EARN_ERR_TIMEOUT
    B.earn_workspace_init(ses.workspace)
    assert bud.device_status() == B.EARN_OK


def test_steps_after_the_packed_prompt_is_gone():
    """Released layers free the packed K/V and decode as unreleased ones do."""
    w = wl.Workload("release", batch=2, n_layers=1, split_k=1, n_q_heads=8, n_kv_heads=8, head_dim=128, dtype="bf16", prompt_len=0,
                    lens=(900, 1200), r_head=4, r_tail=4, decode_steps=3, seed=5)
    total, outs = int(wl.cu_seqlens(w)[-1]), []
    for release in (False, True):
        ses = make_session(w)
        bud = BudgetedLayers(ses, 64)
        q, k, v = wl.layer_qkv(w, 0, "cuda")
        lse = torch.empty(w.n_q_heads, total, device="cuda")
        ses.prefill_layer(0, q, k, v, lse=lse)
        bud.take_prompt(0, q, k, v, lse, release=release)
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        del k, v
        freed = before - torch.cuda.memory_allocated()
        assert freed == (2 * total * 8 * 128 * 2 if release else 0)
        junk = torch.full((2 * total, 8, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
        out = []
        for step in range(1, 4):
            bud.begin_step()
            out.append(bud.decode_layer(0, *wl.decode_qkv(w, 0, step, "cuda")))
            bud.end_step()
        outs.append(torch.stack(out))
        del junk
    assert torch.equal(*outs)
