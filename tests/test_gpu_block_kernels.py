"""Every kernel that the feed-forward block's calls choose between, against 64 bits: each output tile of the 4-bit
products at lengths of K around its stages and around four k tiles, each tile of the gated block by each output that it
has, whole and in slices of K, and the decode step's column groups by its row tiles.  Which kernel a size takes is
asked for, workspaces are full of NaN, and what lies around an output stays as it was."""
import numpy as np
import pytest

import block_reference as ref
from paper_2603_15965_amd import binding as mb

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh"]


def _normal(torch, seed, *shape, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()


def _operands(torch, N, d_in, d_out, C, rank):
    x, W = _normal(torch, N, N, d_in), _normal(torch, d_in, d_in, d_out, std=d_in ** -0.5)
    if C == 0:
        return x, W, None, None, None
    A, B = _normal(torch, C, C, d_in, rank, std=d_in ** -0.5), _normal(torch, rank, C, rank, d_out, std=0.25 * rank ** -0.5)
    r = np.random.default_rng(N + C).integers(0, C, N)
    r[C % 5::17], r[0::23] = -1, C + 1
    return x, W, A, B, torch.from_numpy(r.astype(np.int32)).cuda()


def _guarded(torch, shape, dtype):
    n = int(np.prod(shape))
    room = torch.full((n + 512,), 7.0, dtype=dtype, device="cuda")
    return room[256:256 + n].view(shape), lambda: bool((room[:256] == 7).all() and (room[256 + n:] == 7).all())


def _nan_workspace(torch, fn, *sizes):
    """A workspace of NaN between guards."""
    n = int(getattr(mb.load(), fn)(*sizes))
    room = torch.full((n + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    return room[256:256 + n], lambda: bool((room[:256] == 0xFF).all() and (room[256 + n:] == 0xFF).all())


# ---- products on a 4-bit weight ----

T256, T256W, T128, T128D, T64W, T64 = (256, 256, 4), (256, 128, 3), (128, 128, 3), (128, 128, 4), (64, 128, 4), (64, 64, 4)
# (by tile; k tiles of 128 are 1 .. 13: fewer than the stages, as many, a multiple of four and not)
PRODUCTS = [(T64, s) for s in ((65, 72, 72), (65, 136, 72), (65, 264, 72), (66, 392, 72), (67, 520, 72), (65, 648, 72), (66, 776, 72),
                               (65, 920, 72), (66, 1032, 72), (66, 1288, 72), (65, 1544, 72))]
PRODUCTS += [(T64W, s) for s in ((13665, 72, 328), (13646, 136, 328), (14726, 264, 328), (8133, 392, 584), (13703, 528, 328),
                                 (396, 784, 10440), (325, 920, 11464), (340, 1048, 10872), (15116, 1296, 200))]
PRODUCTS += [(T128, s) for s in ((961, 72, 10472), (14953, 136, 648), (706, 272, 11080), (3667, 392, 2184), (14221, 528, 520),
                                 (8268, 648, 904), (9357, 776, 776), (10965, 904, 664), (10953, 1048, 648))]
PRODUCTS += [(T128D, s) for s in ((14376, 528, 2696), (8055, 648, 1928), (13029, 784, 520), (12324, 904, 520), (14520, 1032, 392))]
PRODUCTS += [(T256W, s) for s in ((15314, 264, 904), (15359, 400, 808), (15015, 528, 776), (13967, 656, 808), (14316, 776, 792),
                                  (9957, 904, 1176), (12439, 1032, 920), (12284, 1552, 904))]
PRODUCTS += [(T256, s) for s in ((4067, 1016, 4040), (1987, 1064, 8184), (16323, 1232, 1016), (4046, 1576, 3976))]
# at most 64 tokens: column groups of 16, 32 and 48 by row tiles of 16, one round of 512 k to a wavefront and two
PRODUCTS += [(((N + 15) // 16 * 16, cols, 0), (N, d_in, d_out)) for cols, d_out in ((16, 72), (16, 4088), (32, 4104), (32, 8184), (48, 8200), (48, 8904))
             for N, d_in in ((1, 72), (9, 1032), (16, 4616), (24, 264), (41, 136), (48, 4104), (64, 520))]
RANKS = [8, 16, 24, 40, 64, 72, 128]


@pytest.mark.parametrize("i", range(len(PRODUCTS)), ids=["-".join(map(str, s)) for _, s in PRODUCTS])
def test_products_on_a_4bit_weight(i):
    import torch
    import block_device as dev
    tile, (N, d_in, d_out) = PRODUCTS[i]
    C, rank = (1, 3, 7, 20, 70)[i % 5], RANKS[i % 7]
    print(f"{N} x {d_in} -> {d_out}, tile {tile}, {C} adapters of rank {rank}", flush=True)
    assert mb.molora_mx_matmul_tile(N, d_in, d_out) == tile
    x, W, A, B, r = _operands(torch, N, d_in, d_out, C, rank)
    x[:, d_in // 2] *= 30     # blocks of very different scales
    wc, ws = mb.molora_mx_quantize_w(W)
    xc, xs = mb.molora_mx_quantize(x)
    qx, qw = mb.molora_mx_dequantize(xc, xs, N, d_in).double(), mb.molora_mx_dequantize(wc, ws, d_out, d_in).double()
    rows = np.random.default_rng(i).choice(N, min(N, 16), replace=False)
    assert np.array_equal(qx[rows].cpu().numpy(), ref.mx_values(x[rows].double().cpu().numpy()))
    want, off = dev.mm(qx, qw.t()), (d_in + 1) * ref.ULP32 * dev.mm(qx.abs(), qw.abs().t())
    h, h_ok = _guarded(torch, (N, d_out), torch.float32)
    mb.molora_mx_matmul(xc, xs, wc, ws, N, d_in, d_out, h)
    assert h_ok() and bool(((h.double() - want).abs() <= off).all())
    work, work_ok = _nan_workspace(torch, "molora_apply_mx_workspace_bytes", N, d_in, d_out, C, rank)
    h.fill_(7.0)
    mb.molora_apply_mx(x, wc, ws, A, B, r, h, workspace=work)
    l, lo = dev.lora(x.double(), A.double(), B.double(), r)
    off += lo + 2 * ref.ULP32 * (l.abs() + want.abs())
    assert h_ok() and work_ok() and bool(((h.double() - want - l).abs() <= off).all())
    again = torch.empty_like(h)
    mb.molora_apply_mx(x, wc, ws, A, B, r, again, workspace=work)   # on what the call before has left there
    assert torch.equal(again, h)


# ---- the gated block ----

# kernel (rows, columns, stages; None: streaming), in slices or whole, sizes
G64, G128M, G128, G128W, G192, G256, G320 = (64, 128, 3), (128, 128, 4), (128, 128, 2), (128, 256, 3), (192, 256, 2), (256, 256, 2), (320, 256, 2)
GATED = [
    (None, 1, (66, 72, 72, 11, 32)), (None, 1, (300, 264, 520, 30, 64)), (None, 1, (381, 256, 512, 29, 64)),
    (G64, 1, (66, 72, 72, 8, 16)), (G128M, 1, (67, 72, 72, 4, 40)), (G128, 1, (16324, 72, 80, 6, 24)), (G128W, 1, (130, 1104, 12048, 6, 16)),
    (G192, 1, (261, 72, 10896, 6, 16)), (G256, 1, (386, 72, 10936, 6, 40)), (G320, 1, (537, 72, 10960, 3, 8)),
    (G256, 1, (6005, 776, 1048, 80, 16)), (G320, 1, (5003, 328, 1592, 13, 40)),
    (G64, 0, (68, 784, 72, 7, 24)), (G128M, 0, (66, 1304, 72, 8, 128)), (G128, 0, (65, 784, 5536, 10, 128)), (G128W, 0, (68, 4504, 5560, 5, 8)),
    (G192, 0, (137, 4008, 5744, 11, 128)),
    (G64, 1, (66, 72, 72, 0, 0)), (G128M, 1, (16367, 144, 72, 0, 0)), (G128, 1, (16324, 72, 80, 0, 0)), (G128W, 1, (134, 1064, 11312, 0, 0)),
    (G192, 1, (13065, 72, 264, 0, 0)), (G256, 1, (386, 72, 10936, 0, 0)), (G320, 1, (533, 72, 12152, 0, 0)),
    (G64, 0, (66, 1272, 72, 0, 0)), (G128M, 0, (66, 4040, 1776, 0, 0)), (G128, 0, (65, 3784, 5448, 0, 0)), (G128W, 0, (65, 4272, 5464, 0, 0)),
    (G192, 0, (130, 7112, 4184, 0, 0)),
]


def _forward(torch, dev, sizes, act):
    N, d_in, F, C, rank = sizes
    args = _operands(torch, N, d_in, 2 * F, C, rank)
    wide = [None if t is None else t.double() if t.is_floating_point() else t for t in args]
    h, off = dev.projection(*wide)
    want, z_off = dev.act(h[:, :F], act)[0] * h[:, F:], dev.gated_off(h, off, act)
    work, work_ok = _nan_workspace(torch, "molora_apply_gated_workspace_bytes", N, d_in, F, C, rank)
    z, z_ok = _guarded(torch, (N, F), torch.bfloat16)
    pre, pre_ok = _guarded(torch, (N, 2 * F), torch.float32)
    mb.molora_apply_gated(*args, act=act, z=z, pre=pre, workspace=work)
    assert z_ok() and pre_ok() and work_ok()
    assert bool(((pre.double() - h).abs() <= off).all()), "h"
    assert bool(((z.double() - want).abs() <= z_off).all()), "z with h"
    alone, alone_ok = _guarded(torch, (N, F), torch.bfloat16)
    mb.molora_apply_gated(*args, act=act, z=alone, workspace=work)
    assert alone_ok() and work_ok() and torch.equal(alone, z), "z without h"
    return args, wide, pre


@pytest.mark.parametrize("i", range(len(GATED)), ids=["-".join(map(str, s)) for _, _, s in GATED])
def test_gated_block(i):
    import torch
    import block_device as dev
    tile, whole, sizes = GATED[i]
    print(f"gated {sizes}, tile {tile}", flush=True)
    got = mb.molora_apply_gated_tile(*sizes)
    assert (got[3] == 1) == bool(whole) and (got[2] == 0 if tile is None else got[:3] == tile), got
    _forward(torch, dev, sizes, ACTS[i % 3])


@pytest.mark.parametrize("N", [1, 7, 24, 33, 48, 64])
@pytest.mark.parametrize("d_in,F,cols", [(136, 72, 32), (264, 4088, 32), (1032, 4120, 64), (72, 8184, 64), (520, 8200, 128), (4104, 8328, 128)])
@pytest.mark.parametrize("C,rank", [(0, 0), (5, 40), (70, 16)])
def test_gated_block_of_few_tokens(N, d_in, F, cols, C, rank):
    import torch
    import block_device as dev
    print(f"gated {N} x {d_in} -> 2 x {F}, {C} of rank {rank}", flush=True)
    assert mb.molora_apply_gated_tile(N, d_in, F, C, rank)[:3] == ((N + 15) // 16 * 16, cols, 0)
    _forward(torch, dev, (N, d_in, F, C, rank), ACTS[(N + F + C) % 3])


# by the kernel of dx, then by that of dW
DX = [(G64, 1, (66, 72, 72, 8, 16)), (G128M, 1, (66, 72, 72, 11, 32)), (G128, 1, (10922, 264, 72, 7, 72)), (G128W, 1, (9149, 400, 672, 9, 8)),
      (G192, 1, (13335, 520, 72, 10, 8)), (G256, 1, (16353, 560, 72, 8, 72)), (G320, 1, (16379, 816, 72, 4, 8)),
      (G64, 0, (68, 72, 272, 6, 64)), (G128M, 0, (66, 72, 264, 10, 72)), (G128, 0, (65, 11176, 424, 10, 128)), (G128W, 0, (68, 11408, 2160, 4, 24)),
      (G192, 0, (131, 11472, 1960, 11, 128))]
DW = [(G64, 1, (66, 72, 72, 11, 32)), (G128M, 1, (139, 200, 8176, 7, 64)), (G128, 1, (66, 11056, 136, 10, 40)), (G128W, 1, (1046, 136, 11408, 4, 128)),
      (G192, 1, (67, 528, 6752, 11, 64)), (G256, 1, (66, 392, 11056, 12, 72)), (G320, 1, (65, 528, 12264, 3, 16)),
      (G64, 0, (1227, 72, 72, 8, 128)), (G128M, 0, (3846, 1880, 72, 6, 24)), (G128, 0, (4103, 5488, 72, 7, 16)), (G128W, 0, (4442, 5384, 72, 0, 0)),
      (G192, 0, (5736, 136, 5520, 10, 128))]


@pytest.mark.parametrize("i", range(len(DX) + len(DW)), ids=["dx-" * (k < len(DX)) + "dW-" * (k >= len(DX)) + "-".join(map(str, s))
                                                            for k, (_, _, s) in enumerate(DX + DW)])
def test_gradients(i):
    import torch
    import block_device as dev
    tile, whole, sizes = (DX + DW)[i]
    N, d_in, F, C, rank = sizes
    act = ACTS[i % 3]
    print(f"gated backward {sizes}, tile {tile}", flush=True)
    got = mb.molora_gated_backward_tile(*sizes)[0 if i < len(DX) else 1]
    assert got[:3] == tile and (got[3] == 1) == bool(whole), got
    args, wide, pre = _forward(torch, dev, sizes, act)
    dz = _normal(torch, F, N, F)
    work, work_ok = _nan_workspace(torch, "molora_gated_backward_workspace_bytes", N, d_in, F, C, rank)
    shapes = {"dx": (N, d_in), "dW": (d_in, 2 * F)} | ({"dA": (C, d_in, rank), "dB": (C, rank, 2 * F)} if C else {})
    bufs = {k: _guarded(torch, s, torch.bfloat16) for k, s in shapes.items()}
    mb.molora_gated_backward(dz, *args, pre, act=act, workspace=work, **{k: b[0] for k, b in bufs.items()})
    assert work_ok()
    for k, (v, off) in dev.gradients(dz.double(), *wide, act).items():
        g = bufs[k][0].double()
        assert bufs[k][1](), f"{k}: written beyond its end"
        assert bool(((g - v).abs() <= off).all()), f"{k}: {float(((g - v).abs() / off.clamp(min=1e-300)).max())} of the bound"
        # two roundings to bf16, each off by at most 2^-8 / sqrt(3) in the mean square
        assert float((g - v).norm()) <= ref.HALF16 * float(v.norm()), k
