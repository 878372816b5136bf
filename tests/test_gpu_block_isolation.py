"""What one adapter holds reaches its own tokens only: infinities and NaN in the A and B of one adapter change no bit
of another adapter's rows, of a row without adapter, or of another adapter's gradients, in every kernel of the
feed-forward block that multiplies rows of several adapters by turns."""
import numpy as np
import pytest

from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _case(N, d_in, d_out, C, rank):
    import torch
    from paper_2603_15965_amd import binding as mb
    w = wl.custom("own", N, d_in, d_out, C, rank, wl.BASE_SEED + 61000 + N + d_in)
    r = np.random.default_rng(N).integers(0, C, N).astype(np.int32)
    r[2::7], r[5::11] = -1, C + 2
    r[0] = 1   # the adapter to be spoiled is in use
    if N < 3:
        r[1:] = 0
    x, W, A, B = (mb.bf16_tensor(t) for t in (w.x, w.W, w.A, w.B))
    return torch, mb, x, W, A, B, r, torch.from_numpy(r).cuda()


def _spoiled(A, B, c):
    A2, B2 = A.clone(), B.clone()
    A2[c, 0, 0], A2[c, A.shape[1] // 2, :] = float("inf"), float("nan")
    B2[c, -1, ::3], B2[c, 0, 1::5], B2[c, 0, -1] = float("inf"), float("nan"), float("-inf")
    return A2, B2


def _same_but(torch, a, b, own):
    """Rows that are not `own` have the same bits, those that are hold something that is not finite."""
    other = torch.from_numpy(np.flatnonzero(~own)).cuda()
    mine = torch.from_numpy(np.flatnonzero(own)).cuda()
    assert torch.equal(a[other], b[other])
    assert bool((~torch.isfinite(b[mine].float())).any(1).all())


@pytest.mark.parametrize("N,d_in,d_out,C,rank", [
    (2, 136, 72, 2, 8), (9, 264, 72, 4, 24), (33, 136, 5000, 3, 16), (48, 72, 5000, 6, 40), (64, 264, 8904, 16, 64), (64, 72, 520, 4, 128),
    (66, 392, 72, 3, 8), (300, 520, 264, 12, 40),             # 64 x 64 tiles
    (13665, 72, 328, 5, 16), (961, 72, 10472, 40, 24),        # 64 x 128, 128 x 128
    (13029, 784, 520, 7, 72),                                 # 128 x 128 of four stages
    (15314, 264, 904, 9, 16), (4067, 1016, 4040, 70, 32)])    # 256 x 128, 256 x 256
def test_4bit_projection(N, d_in, d_out, C, rank):
    print(f"apply_mx, a spoiled adapter: {N} x {d_in} -> {d_out}, {C} of rank {rank}", flush=True)
    torch, mb, x, W, A, B, r, rd = _case(N, d_in, d_out, C, rank)
    wc, ws = mb.molora_mx_quantize_w(W)
    A2, B2 = _spoiled(A, B, 1)
    h = mb.molora_apply_mx(x, wc, ws, A, B, rd)
    h2 = mb.molora_apply_mx(x, wc, ws, A2, B2, rd)
    assert bool(torch.isfinite(h).all())
    _same_but(torch, h, h2, r == 1)


@pytest.mark.parametrize("N,d_in,F,C,rank", [
    (2, 136, 72, 2, 8), (9, 136, 40, 3, 16), (17, 64, 5000, 4, 24), (64, 136, 8904, 16, 40), (50, 72, 520, 4, 128),
    (66, 72, 72, 11, 32), (300, 264, 520, 30, 64),            # the streaming kernel
    (69, 72, 72, 8, 16), (68, 784, 72, 7, 24),                # 64 x 128 tiles, in one launch and in slices of K
    (67, 72, 72, 4, 40), (66, 1304, 72, 8, 128),              # 128 x 128
    (16324, 72, 80, 6, 24), (65, 784, 5536, 10, 128),         # 128 x 128 of two stages
    (130, 1104, 12048, 6, 16), (68, 4504, 5560, 5, 8),        # 128 x 256
    (261, 72, 10896, 6, 16), (137, 4008, 5744, 11, 128),      # 192 x 256
    (386, 72, 10936, 6, 40), (537, 72, 10960, 3, 8)])         # 256 x 256, 320 x 256
def test_gated_block(N, d_in, F, C, rank):
    print(f"gated, a spoiled adapter: {N} x {d_in} -> 2 x {F}, {C} of rank {rank}", flush=True)
    torch, mb, x, W, A, B, r, rd = _case(N, d_in, 2 * F, C, rank)
    A2, B2 = _spoiled(A, B, 1)
    pre, pre2 = (torch.empty(N, 2 * F, dtype=torch.float32, device="cuda") for _ in range(2))
    z = mb.molora_apply_gated(x, W, A, B, rd, pre=pre)
    z2 = mb.molora_apply_gated(x, W, A2, B2, rd, pre=pre2)
    assert bool(torch.isfinite(pre).all())
    _same_but(torch, z, z2, r == 1)
    _same_but(torch, pre, pre2, r == 1)
    assert torch.equal(mb.molora_apply_gated(x, W, A, B, rd), z)


@pytest.mark.parametrize("N,d_in,F,C,rank", [
    (9, 136, 40, 3, 16), (64, 72, 264, 5, 64),
    (66, 72, 72, 8, 16), (68, 72, 272, 6, 64),                # 64 x 128 tiles, in one launch and in slices of K
    (66, 72, 72, 11, 32), (66, 72, 264, 10, 72),              # 128 x 128
    (10922, 264, 72, 7, 72), (65, 11176, 424, 10, 128),       # 128 x 128 of two stages
    (9149, 400, 672, 9, 8), (68, 11408, 2160, 4, 24),         # 128 x 256
    (13335, 520, 72, 10, 8), (131, 11472, 1960, 11, 128),     # 192 x 256
    (16353, 560, 72, 8, 72), (16379, 816, 72, 4, 8)])         # 256 x 256, 320 x 256
def test_gradients(N, d_in, F, C, rank):
    print(f"gated backward, a spoiled adapter: {N} x {d_in} -> 2 x {F}, {C} of rank {rank}", flush=True)
    torch, mb, x, W, A, B, r, rd = _case(N, d_in, 2 * F, C, rank)
    A2, B2 = _spoiled(A, B, 1)
    pre = torch.empty(N, 2 * F, dtype=torch.float32, device="cuda")
    mb.molora_apply_gated(x, W, A, B, rd, pre=pre)
    g = torch.Generator(device="cuda").manual_seed(N)
    dz = torch.randn(N, F, generator=g, device="cuda").bfloat16()
    clean = mb.molora_gated_backward(dz, x, W, A, B, rd, pre)
    got = mb.molora_gated_backward(dz, x, W, A2, B2, rd, pre)
    assert all(bool(torch.isfinite(t.float()).all()) for t in clean)
    _same_but(torch, clean[0], got[0], r == 1)
    assert torch.equal(clean[1], got[1])   # dW has no adapter in it
    for a, b in zip(clean[2:], got[2:]):
        keep = [c for c in range(C) if c != 1]
        assert torch.equal(a[keep], b[keep]) and not bool(torch.isfinite(b[1].float()).all())


@pytest.mark.parametrize("N,d_in,F,C,rank", [(2, 72, 72, 2, 8), (33, 264, 40, 3, 16), (64, 136, 4120, 5, 40), (66, 72, 72, 11, 32),
                                             (300, 264, 520, 4, 24), (515, 520, 264, 7, 16), (2056, 72, 136, 70, 8)])
def test_rows_that_are_not_finite(N, d_in, F, C, rank):
    """A row of x, and a value of dz, reach their own row and the gradients that sum over it, no other row or adapter."""
    print(f"spoiled rows: {N} x {d_in} -> 2 x {F}, {C} of rank {rank}", flush=True)
    torch, mb, x, W, A, B, r, rd = _case(N, d_in, 2 * F, C, rank)
    rows = np.zeros(N, bool)
    rows[[0, N - 1]] = True
    x2 = x.clone()
    x2[0, d_in - 1], x2[N - 1, 0] = float("inf"), float("nan")
    pre, pre2 = (torch.empty(N, 2 * F, dtype=torch.float32, device="cuda") for _ in range(2))
    z = mb.molora_apply_gated(x, W, A, B, rd, pre=pre)
    z2 = mb.molora_apply_gated(x2, W, A, B, rd, pre=pre2)
    _same_but(torch, z, z2, rows)
    _same_but(torch, pre, pre2, rows)
    wc, ws = mb.molora_mx_quantize_w(W)
    _same_but(torch, mb.molora_apply_mx(x, wc, ws, A, B, rd), mb.molora_apply_mx(x2, wc, ws, A, B, rd), rows)
    g = torch.Generator(device="cuda").manual_seed(N)
    dz = torch.randn(N, F, generator=g, device="cuda").bfloat16()
    dz2 = dz.clone()
    dz2[0, F - 1] = float("nan")
    clean, got = (mb.molora_gated_backward(t, x, W, A, B, rd, pre) for t in (dz, dz2))
    rows[N - 1] = False
    _same_but(torch, clean[0], got[0], rows)
    keep = [c for c in range(C) if c != r[0]]
    assert torch.equal(clean[2][keep], got[2][keep]) and torch.equal(clean[3][keep], got[3][keep])
    assert not bool(torch.isfinite(got[1].float()).all())
