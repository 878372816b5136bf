"""Memory that the feed-forward block's calls allocate by themselves: outputs and workspaces on a stream other than the
current one, and of calls that a graph records."""
import numpy as np
import pytest

from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu
N, D, F, C, RANK = 300, 264, 520, 4, 16


@pytest.fixture(scope="module")
def block():
    """The calls as {name: f(stream)}, each with its outputs in a tuple, and the number of the first that it allocates."""
    import torch
    from paper_2603_15965_amd import binding as mb
    w = wl.custom("gated", N, D, 2 * F, C, RANK, 7100 + wl.BASE_SEED)
    x, W, A, B = (mb.bf16_tensor(t) for t in (w.x, w.W, w.A, w.B))
    r = torch.from_numpy(w.r).cuda()
    dz = mb.bf16_tensor(wl.normal_bf16(7101, (N, F), 1.0))
    pre = torch.empty(N, 2 * F, dtype=torch.float32, device="cuda")
    mb.molora_apply_gated(x, W, A, B, r, pre=pre)
    xc, xs = mb.molora_mx_quantize(x)
    wc, ws = mb.molora_mx_quantize_w(W)
    torch.cuda.synchronize()
    return {
        "mx_quantize": lambda s: mb.molora_mx_quantize(x, stream=s),
        "mx_quantize_w": lambda s: mb.molora_mx_quantize_w(W, stream=s),
        "mx_dequantize": lambda s: (mb.molora_mx_dequantize(xc, xs, N, D, stream=s),),
        "mx_matmul": lambda s: (mb.molora_mx_matmul(xc, xs, wc, ws, N, D, 2 * F, stream=s),),
        "apply_mx": lambda s: (mb.molora_apply_mx(x, wc, ws, A, B, r, stream=s),),
        "apply_gated": lambda s: (mb.molora_apply_gated(x, W, A, B, r, stream=s),),
        "gated_backward": lambda s: mb.molora_gated_backward(dz, x, W, A, B, r, pre, stream=s),
    }


@pytest.mark.parametrize("name", ["mx_quantize", "mx_quantize_w", "mx_dequantize", "mx_matmul", "apply_mx", "apply_gated", "gated_backward"])
@pytest.mark.parametrize("as_number", [False, True])
def test_outputs_are_not_memory_that_the_current_stream_still_uses(block, name, as_number):
    """The current stream is busy, will then write to tensors of the outputs' sizes, and the host has given these
    back already: the call on a side stream must not be handed their memory."""
    import torch
    call = block[name]
    want = call(None)
    big = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    out = torch.empty_like(big)
    call(side)   # (what the side stream needs from the runtime is there)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    gone = [torch.empty_like(t) for t in want]
    torch.cuda.synchronize()
    print(f"{name} on a side stream", flush=True)
    for _ in range(20):   # some milliseconds
        torch.mm(big, big, out=out)
    for t in gone:
        t.fill_(77)
    del gone, t
    got = call(side.cuda_stream if as_number else side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["mx_quantize", "mx_matmul", "apply_mx", "apply_gated", "gated_backward"])
def test_memory_of_a_recorded_call_belongs_to_the_graph(block, name):
    """A call recorded without outputs and workspace: what it writes on every replay is handed to nobody else,
    whether or not the caller has kept its outputs."""
    import torch
    from paper_2603_15965_amd import binding as mb
    call = block[name]
    want = call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    call(side)   # the side stream has the memory, given back
    side.synchronize()
    print(f"{name} recorded", flush=True)
    g, kept = mb.Graph(side), mb.Graph(side)
    with g.capture():
        call(side)
    with kept.capture():
        got = call(side)
    with torch.cuda.stream(side):   # all that is free on the stream, of any size that the call can have asked for
        fresh = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (1 << 12, 1 << 15, 1 << 18, 1 << 20, 5 << 20) for _ in range(3)]
    for replay in range(3):
        for t in got:
            t.fill_(99)
        torch.cuda.synchronize()
        g.launch()
        kept.launch()
        side.synchronize()
        assert all(bool((t == 7).all()) for t in fresh), f"replay {replay} wrote to memory that is another tensor's"
        for a, b in zip(got, want):
            assert torch.equal(a, b), f"replay {replay}"
    g.destroy()
    kept.destroy()
