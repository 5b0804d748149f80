"""PagedLayers against the calls it is made of, bit for bit, and captured: a step's graph replayed with other target lengths gives
what uncaptured steps give."""
import numpy as np
import pytest
import torch

from paper_2507_00715_b200 import binding as B
from paper_2507_00715_b200.rope import frequencies
from paper_2507_00715_b200.session import PagedLayers
from test_gpu_step import DT, gen, i32

pytestmark = pytest.mark.gpu
SPLIT, HQ, HKV, D, ROOM, PAGES, LONGEST = 2, 8, 2, 128, 160, 40, 300
STEPS = ([100, 0, 37], [101, 60, 37], [160, 61, 40], [150, 62, 0], [151, 62, 33], [300, 200, 300], [152, 0, 34])


def layers(dtype):
    f, amp = frequencies(D, scaling="ramp", factor=4.0, original=128)
    return PagedLayers(3, SPLIT, HQ, HKV, D, DT[dtype], 3, PAGES, LONGEST, ROOM, f, False, amp)


def inputs(dtype):
    g = gen(5)
    return [[torch.randn(ROOM, HQ + 2 * HKV, D, generator=g, device="cuda").to(DT[dtype]) for _ in range(SPLIT)] for _ in STEPS]


def parts(qkv):
    return qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]


def state(lay):
    live = int(lay.n_free)
    return [lay.held, lay.seq_len, lay.cu_new, lay.n_free, lay.n_refused, lay.positions, lay.slots, lay.block_table, lay.free_pages[:live],
            *lay.k_pages, *lay.v_pages]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_calls_it_is_made_of(dtype):
    lay, raw, data = layers(dtype), layers(dtype), inputs(dtype)
    refused = 0
    for target, qkv in zip(STEPS, data):
        lay.begin_step(i32(target))
        B.earn_page_tables(3, i32(target), raw.pool, raw.step, raw.held, raw.n_free, raw.table_workspace)
        for layer in range(SPLIT):
            lse = torch.zeros(HQ, ROOM, device="cuda")
            got = lay.layer(layer, *parts(qkv[layer]), lse=lse)
            o, other = torch.zeros_like(got), torch.zeros_like(lse)
            B.earn_rope_append(raw.model, layer, raw.rope, ROOM, raw.positions, raw.slots, *parts(qkv[layer]), raw.q_turned, raw.caches[layer])
            B.earn_paged_chunk_attn(raw.model, 3, layer, ROOM, raw.cu_new, raw.q_turned, raw.caches[layer], o, other, raw.workspace)
            assert torch.equal(got, o) and torch.equal(lse, other)
        assert all(torch.equal(x, y) for x, y in zip(state(lay), state(raw)))
        assert lay.device_status() == B.EARN_OK and lay.kv_entries() == SPLIT * int(lay.held.sum())
        refused += lay.refused()
    assert refused > 0                                     # (the step that wants more than there is is among them)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured(dtype):
    lay, plain, data = layers(dtype), layers(dtype), inputs(dtype)
    target, qkv = i32([0, 0, 0]), [torch.zeros_like(x) for x in data[0]]
    outs = [torch.zeros(ROOM, HQ, D, device="cuda", dtype=DT[dtype]) for _ in range(SPLIT)]

    def step():
        lay.begin_step(target)
        for layer in range(SPLIT):
            lay.layer(layer, *parts(qkv[layer]), out=outs[layer])

    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()                                             # (nothing held, nothing new)
        with torch.cuda.graph(graph, stream=s):
            step()
        for lengths, x in zip(STEPS, data):
            target.copy_(i32(lengths))
            for layer in range(SPLIT):
                qkv[layer].copy_(x[layer])
                outs[layer].zero_()
            graph.replay()
            plain.begin_step(i32(lengths))
            for layer in range(SPLIT):
                assert torch.equal(outs[layer], plain.layer(layer, *parts(x[layer])))
            assert all(torch.equal(a, b) for a, b in zip(state(lay), state(plain)))
            assert lay.device_status() == B.EARN_OK
    torch.cuda.current_stream().wait_stream(s)
    assert np.asarray(STEPS).max() <= LONGEST
