"""Orders, captures and values at the edges of what the calls around the projection allow."""
import math

import pytest
import torch

import around_ref as ref
from paper_2603_05035_b200 import binding
from test_gpu_around_projection import filled, rnd

pytestmark = pytest.mark.gpu
DT = ref.DT


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    c.ensure_attention_workspace()
    yield c
    c.close()


# ---- scratch of the attention ---------------------------------------------------------------------

def long_attention(seed=60):
    """One sequence whose heads are cut into parts, so that scratch is used: the call, its result and what it has to be."""
    paged, _ = filled(seed, [9000], 16, 2, 64, "token", "bf16")
    Q, ln = rnd(seed + 1, 1, 8 * 64, dtype="bf16"), torch.tensor([9000], dtype=torch.int32, device="cuda")
    other = binding.Context(0)
    other.ensure_attention_workspace()
    want, o = torch.empty_like(Q), torch.zeros_like(Q)
    other.paged_attention(paged, Q, ln, want)
    torch.cuda.synchronize()
    other.close()
    return (lambda c: c.paged_attention(paged, Q, ln, o)), o, want


def captured(call, c):
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c)
    return graph


def test_attention_leaves_the_batches_workspace_alone():
    """A replay cannot hold back a batch, so it must not write where batches sample, whichever workspace was set first and however large."""
    call, o, want = long_attention()
    for first in (True, False):
        c = binding.Context(0)
        ws = torch.full((16 << 20,), 0x5A, dtype=torch.uint8, device="cuda")
        if first:
            c.set_workspace(ws)
        c.ensure_attention_workspace()
        if not first:
            c.set_workspace(ws)
        graph = captured(call, c)
        graph.replay()
        call(c)
        torch.cuda.synchronize()
        assert (ws == 0x5A).all() and torch.equal(o, want)
        c.close()


def test_replayed_attention_between_two_batches():
    """Batch, replay and batch of the same shape on one stream, against the same with waits in between."""
    n, k, d, p, calls = 512, 26, 512, 1536, 4
    c = binding.Context(0)
    c.set_lanes(calls)
    c.ensure_batch_workspace(n, k, d, p, "bf16", calls)
    c.ensure_attention_workspace()
    call, o, want = long_attention(62)
    H = [rnd(64 + i, n, d, dtype="bf16") for i in range(calls)]
    W = [rnd(70, d, p, scale=0.02, dtype="bf16")] * calls

    def run(between):
        outs = []
        graph = captured(call, c)
        o.zero_()
        for step in range(6):
            q = [torch.empty((n, p), dtype=torch.bfloat16, device="cuda") for _ in range(calls)]
            between()
            c.qkv_offload_batch(H, W, n, k, d, p, [binding.ORTHOGONAL] * calls, [100 * step + i for i in range(calls)], 10.0, "bf16", q)
            between()
            graph.replay()
            between()
            outs += q + [o.clone()]
        torch.cuda.synchronize()
        return outs

    apart = run(torch.cuda.synchronize)
    close = run(lambda: None)
    assert all(torch.equal(a, b) for a, b in zip(apart, close)) and torch.equal(o, want)
    assert c.last_status() == binding.OK
    c.close()


def test_captured_attention_outlives_a_larger_workspace():
    """A later call that needs a larger workspace lets go of the old one; what was captured before does not use it."""
    c = binding.Context(0)
    c.ensure_attention_workspace()
    call, o, want = long_attention(66)
    graph = captured(call, c)
    c.set_workspace(torch.empty(12 << 20, dtype=torch.uint8, device="cuda"))
    c.ensure_workspace(512, 26, 512, 1536, "bf16")
    c.set_workspace(None)
    taken = [torch.full((12 << 20,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and all((t == 0x5A).all() for t in taken)
    c.close()


def test_attention_in_the_shared_workspace():
    """Without scratch of its own a call works in the general workspace, unless it is being captured."""
    call, o, want = long_attention(68)
    c = binding.Context(0)
    c.set_workspace(torch.empty(c._lib.gelo_attention_workspace_bytes(), dtype=torch.uint8, device="cuda"))
    call(c)
    torch.cuda.synchronize()
    assert torch.equal(o, want)
    x, graph = torch.zeros(4, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(binding.GeloError) as e:
            call(c)
    assert e.value.status == binding.ERR_WORKSPACE
    c.ensure_attention_workspace()
    o.zero_()
    captured(call, c).replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want)
    c.close()
