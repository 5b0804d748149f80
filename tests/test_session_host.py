"""Host side of the budgeted layers: what a budget has to hold, whose status is reported, what a released prompt leaves."""
import gc
import weakref

import numpy as np
import pytest
import torch

from paper_2507_00715_b200 import binding as B
from paper_2507_00715_b200.session import BudgetedLayers, EarnSession
from test_abi_host import lib  # noqa: F401  (the fixture builds the library)


@pytest.fixture
def session(lib, monkeypatch):  # noqa: F811
    """Two full layers and a register layer, four registers at either end, in host memory (no call reaches a device)."""
    monkeypatch.setattr(B, "earn_workspace_init", lambda workspace: None)
    monkeypatch.setattr(B, "make_paged_cache", lambda *a: a)
    monkeypatch.setattr(B, "earn_paged_workspace_bytes", lambda *a: 256)
    cu = np.concatenate([[0], np.cumsum([30, 9, 50])])
    return EarnSession(3, 2, 4, 2, 64, torch.float32, cu, 4, 4, max_new=6, device="cpu")


def test_a_budget_holds_the_registers_and_the_last_rows(session):
    for budget, n_last, policy, pinned in ((24, None, (24, 4, 4), 4), (10, None, (10, 4, 2), 4), (8, None, (8, 4, 0), 4),
                                           (16, 8, (16, 4, 8), 4), (20, 2, (20, 4, 2), 2), (20, 0, (20, 4, 0), 0)):
        bud = BudgetedLayers(session, budget, n_last=n_last)
        assert (bud.policy.budget, bud.policy.n_first, bud.policy.n_last) == policy
        want = sorted(e - i for e in (30, 39, 89) for i in range(1, pinned + 1))
        assert sorted(bud.pinned_rows.tolist()) == want
    for kw in (dict(budget=7), dict(budget=15, n_last=8), dict(budget=9, n_first=2, n_last=4)):
        with pytest.raises(ValueError, match="does not hold"):
            BudgetedLayers(session, **kw)
    BudgetedLayers(session, 56, n_last=52)   # (nothing reaches it: 50 rows and six steps)


def test_a_timeout_of_the_prompts_weighing_reaches_the_budgeted_layers(session, monkeypatch):
    """earn_key_weights reports into the workspace it is given, which is the session's."""
    bud = BudgetedLayers(session, 24)
    given = []
    for name in ("earn_key_weights", "earn_evict_prompt_kv"):
        monkeypatch.setattr(B, name, lambda *a, name=name: given.append((name, a[-1])))
    bud.take_prompt(0, None, None, None, None)
    word = torch.zeros(1, dtype=torch.int32)
    monkeypatch.setattr(B, "earn_device_status", lambda ws: int(word) if ws is dict(given)["earn_key_weights"] else B.EARN_OK)
    assert bud.device_status() == B.EARN_OK
    word.fill_(B.EARN_ERR_TIMEOUT)
    assert bud.device_status() == B.EARN_ERR_TIMEOUT


def test_the_session_lets_go_of_a_released_prompt(session, monkeypatch):
    """The packed K/V of a full layer are referenced by nobody but the caller after a released take_prompt, the layer's own
    decode is refused, and the accounting follows."""
    for name in ("earn_prefill_attn", "earn_key_weights", "earn_evict_prompt_kv", "earn_decode_attn"):
        monkeypatch.setattr(B, name, lambda *a: None)
    bud = BudgetedLayers(session, 24)
    q, lens = torch.zeros(89, 4, 64), (30, 9, 50)
    kept, held = [], sum(min(n + 2, 24) for n in lens)
    for layer in range(2):
        k, v = torch.zeros(89, 2, 64), torch.zeros(89, 2, 64)
        kept += [weakref.ref(k), weakref.ref(v)]
        session.prefill_layer(layer, q, k, v)
        bud.take_prompt(layer, q, k, v, None, release=layer == 1)
    del k, v
    gc.collect()
    assert [r() is None for r in kept] == [False, False, True, True]
    registers = (8 + 2) * 3
    assert session.kv_entries(2) == 89 + 2 * 3 + registers
    assert bud.kv_entries(2) == 2 * held + 89 + registers
    for layer in (-1, 2):
        with pytest.raises(ValueError, match="not a full layer"):
            session.release_prompt(layer)
    session.decode_layer(0, 1, q[:3], None, None)
    with pytest.raises(ValueError, match="released"):
        session.decode_layer(1, 1, q[:3], None, None)
    session.prefill_layer(1, q, torch.zeros(89, 2, 64), torch.zeros(89, 2, 64))
    session.decode_layer(1, 1, q[:3], None, None)
    assert session.kv_entries(2) == 2 * (89 + 2 * 3) + registers


def test_the_binding_turns_down_workspaces_and_prompt_offsets_it_must_not_pass(monkeypatch):
    """A workspace in host memory, one that is not dense, and offsets of another type never reach the library.  (Host tensors
    stand in for device tensors: their device number is -1.)"""
    called = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or B.EARN_OK

    monkeypatch.setattr(B, "lib", Library)
    monkeypatch.setattr(B, "_stream_of", lambda device: None)
    model, batch = B.make_model(1, 1, 2, 1, 64, "f32"), B.Batch(np.asarray([0, 3, 5]), 0, 0, device="cpu")
    cache = B.EarnPagedCache(0, 0, None, 1, 2, 0, 16)
    cache.kind, cache.n_seq, cache.device = (torch.float32, 1, 64), 2, -1
    f32, i32 = torch.zeros(2048), torch.zeros(64, dtype=torch.int32)

    def calls(ws):
        yield lambda: B.earn_key_weights(model, batch, 0, 4, f32, f32, f32, f32, ws)
        yield lambda: B.earn_evict_prompt_kv(model, batch, 0, B.make_evict(4), f32, f32, f32, cache, f32, i32, ws)
        yield lambda: B.earn_paged_decode_attn(model, 2, 0, f32, None, None, cache, f32, workspace=ws)
        yield lambda: B.earn_evict_kv(model, 2, 0, B.make_evict(4), cache, f32, i32, f32, i32, ws)

    dense = torch.zeros(512, dtype=torch.uint8)
    monkeypatch.setattr(B, "_current_device", lambda: -1)
    for call in calls(dense):
        call()
    assert len(called) == 4
    for call in calls(torch.zeros(2, dtype=torch.uint8).expand(256, 2)):
        with pytest.raises(ValueError, match="workspace"):
            call()
    for bad in (batch.cu_dev.long(), batch.cu_dev[:2], torch.zeros(3, 2, dtype=torch.int32)[:, 0]):
        with pytest.raises(ValueError, match="cu_seqlens"):
            B.Batch(batch.cu_host, 0, 0, cu_seqlens_dev=bad)
    batch.device = 0
    for call in list(calls(dense))[:2]:
        with pytest.raises(ValueError, match="cu_seqlens"):
            call()
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    cache.device = 0
    for call in calls(dense):
        with pytest.raises(ValueError, match="workspace: on cpu"):
            call()
    assert len(called) == 4
