"""The launch timer in the calls of the feed-forward block: the launch that holds the base projection takes it, whichever
kernel that is, and the launches of a backward pass let it pass."""
import pytest

from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _operands(N, d_in, d_out, C, rank):
    import torch
    from paper_2603_15965_amd import binding as mb
    w = wl.custom("timer", N, d_in, d_out, max(C, 1), rank, 5300 + N)
    x, W, A, B = (mb.bf16_tensor(t) for t in (w.x, w.W, w.A, w.B))
    return torch, mb, x, W, ((A, B, torch.from_numpy(w.r).cuda()) if C else (None, None, None))


def _timed(torch, mb, call):
    want = call()
    timer = mb.LaunchTimer()
    for _ in range(2):
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        e0.record()
        timer.arm()
        got = call()
        e1.record()
        torch.cuda.synchronize()
        us = timer.elapsed_us()
        assert 0.5 < us < e0.elapsed_time(e1) * 1e3
        assert torch.equal(got, want)
    timer.destroy()


@pytest.mark.parametrize("N,d_in,F,C,rank", [
    (7, 264, 136, 3, 16), (48, 264, 136, 0, 8),      # at most 64 tokens
    (300, 264, 520, 30, 64),                         # the streaming kernel
    (300, 520, 264, 3, 16), (200, 136, 264, 0, 8),   # the tiled GEMM
    (68, 784, 72, 7, 24)])                           # its slices of K
def test_gated_block(N, d_in, F, C, rank):
    torch, mb, x, W, low = _operands(N, d_in, 2 * F, C, rank)
    print(f"timer, gated {N} x {d_in} -> 2 x {F}, {C} of rank {rank}", flush=True)
    _timed(torch, mb, lambda: mb.molora_apply_gated(x, W, *low))


@pytest.mark.parametrize("N,d_in,d_out,C,rank", [(1, 264, 136, 2, 8), (64, 264, 520, 5, 40), (300, 520, 264, 4, 16)])
def test_4bit_weight(N, d_in, d_out, C, rank):
    torch, mb, x, W, low = _operands(N, d_in, d_out, C, rank)
    print(f"timer, 4-bit weight {N} x {d_in} -> {d_out}", flush=True)
    wc, ws = mb.molora_mx_quantize_w(W)
    xc, xs = mb.molora_mx_quantize(x)
    _timed(torch, mb, lambda: mb.molora_apply_mx(x, wc, ws, *low))
    _timed(torch, mb, lambda: mb.molora_mx_matmul(xc, xs, wc, ws, N, d_in, d_out))


@pytest.mark.parametrize("N", [48, 300])
def test_other_launches_let_it_pass(N):
    """Armed in front of a backward pass, it is taken by the projection that follows."""
    torch, mb, x, W, low = _operands(N, 264, 272, 3, 16)
    pre = torch.empty(N, 272, dtype=torch.float32, device="cuda")
    z = mb.molora_apply_gated(x, W, *low, pre=pre)
    torch.cuda.synchronize()
    timer = mb.LaunchTimer()
    timer.arm()
    mb.molora_gated_backward(z, x, W, *low, pre)
    mb.molora_mx_quantize(x)
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError):
        timer.elapsed_us()
    mb.molora_apply_gated(x, W, *low)
    assert timer.elapsed_us() > 0.5
    timer.destroy()
