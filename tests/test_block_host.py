"""The feed-forward block's operators without a GPU: the reference's own gradients against differences,
sizes, and every refusal of the C ABI and of the binding."""
import ctypes
import os

import numpy as np
import pytest
import torch

import block_reference as ref
from paper_2603_15965_amd import binding as mb

bf, f32, u8, i32 = torch.bfloat16, torch.float32, torch.uint8, torch.int32
EINVAL, EALIGN, EWORKSPACE = -1, -2, -3


@pytest.fixture(scope="module", autouse=True)
def lib():
    from paper_2603_15965_amd import build
    if not os.path.exists(mb.LIB_PATH):
        build.build()
    return mb.load()


@pytest.fixture(scope="module")
def a():
    """A 256-byte aligned address that no refused call reads."""
    buf = (ctypes.c_char * 4096)()
    at = ctypes.addressof(buf)
    yield at + (-at) % 256


# ---- the reference ----

@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_reference_gradients_are_those_of_differences(kind):
    """Central differences in 64 bits with steps of 1e-5 leave 1e-10 of truncation and 1e-11 of rounding."""
    rng = np.random.default_rng(5)
    n, d, F, C, rank = 9, 16, 8, 3, 8
    x, W = rng.standard_normal((n, d)), rng.standard_normal((d, 2 * F)) / 4
    A, B = rng.standard_normal((C, d, rank)) / 4, rng.standard_normal((C, rank, 2 * F)) / 4
    r = np.array([0, 2, -1, 0, 2, 2, 0, 7, 2])   # adapter 1 has no token, two tokens no adapter
    dz = rng.standard_normal((n, F))
    got = ref.gated_gradients(dz, x, W, A, B, r, kind)
    for name, v in (("dx", x), ("dW", W), ("dA", A), ("dB", B)):
        for at in rng.integers(v.size, size=12):
            i = np.unravel_index(at, v.shape)
            keep = v[i]
            side = []
            for s in (1, -1):
                v[i] = keep + s * 1e-5
                side.append((dz * ref.gated(x, W, A, B, r, kind)).sum())
            v[i] = keep
            assert abs((side[0] - side[1]) / 2e-5 - got[name][0][i]) < 1e-7 * (1 + abs(got[name][0][i])), name
    assert not got["dA"][0][1].any() and not got["dB"][0][1].any()


def test_reference_blocks_round_to_the_even_code():
    v = np.zeros((1, 32))
    v[0, :16] = [4, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 5.0001, 7.9, -.25, -.75, -5, -7.9, .2500001, 0]
    codes, X = ref.mx_blocks(v)
    assert X[0, 0] == 0
    assert list(codes[0, 0, :16]) == [6, 0, 2, 2, 4, 4, 6, 6, 7, 7, 8, 10, 14, 15, 1, 0]
    assert ref.mx_blocks(np.full((1, 32), np.inf))[1][0, 0] == 128


# ---- sizes ----

def test_operand_and_workspace_sizes(lib):
    c, s = lib.molora_mx_codes_bytes, lib.molora_mx_scales_bytes
    assert c(1, 8) == 1024 and s(1, 8) == 256
    assert c(17, 136) == 2 * 2 * 1024 and s(17, 520) == 2 * 2 * 256
    assert c(0, 8) == 0 and c(16, 12) == 0 and c(16, 0) == 0 and c(-1, 8) == 0 and c(1 << 30, 1 << 20) == 0
    for f, last in ((lib.molora_apply_mx_workspace_bytes, (640, 8, 16)), (lib.molora_apply_gated_workspace_bytes, (320, 8, 16)),
                    (lib.molora_gated_backward_workspace_bytes, (320, 8, 16))):
        got = [f(n, 512, *last) for n in (0, 1, 7, 8, 9, 63, 64, 65, 100, 511, 512, 513, 4096, 20000)]
        assert got == sorted(got) and got[1] > 0, f
        assert f(16, 512, last[0], 8, 12) == 0 and f(16, 510, *last) == 0 and f(16, 512, last[0], 1025, 8) == 0 and f(-1, 512, *last) == 0
    assert lib.molora_apply_gated_workspace_bytes(300, 512, 320, 0, 0) >= 64 * 640 * 4   # x W of a batch of 64
    assert lib.molora_gated_backward_workspace_bytes(300, 512, 320, 0, 0) > 0
    assert lib.molora_apply_gated_workspace_bytes(300, 512, 320, 0, 8) == 0
    assert lib.molora_apply_gated_workspace_bytes(1 << 20, 2048, 320, 4, 8) == 0   # x of 4 GiB


# ---- refusals of the C ABI: before anything is enqueued ----

def test_mx_entry_points_reject_bad_arguments(lib, a):
    q = lambda src=a, ty=0, c=a, s=a, n=4, k=64: lib.molora_mx_quantize(src, ty, c, s, n, k, None)
    assert q(src=None) == EINVAL and q(ty=2) == EINVAL and q(c=None) == EINVAL and q(k=60) == EINVAL and q(n=-1) == EINVAL
    assert q(src=a + 2) == EALIGN and q(s=a + 8) == EALIGN and q(n=0, src=None, c=None, s=None) == 0
    w = lambda W=a, c=a, s=a, di=64, do=64: lib.molora_mx_quantize_w(W, c, s, di, do, None)
    assert w(W=None) == EINVAL and w(do=60) == EINVAL and w(di=4) == EINVAL and w(c=a + 8) == EALIGN
    d = lambda c=a, dst=a, n=4, k=64: lib.molora_mx_dequantize(c, a, dst, n, k, None)
    assert d(c=None) == EINVAL and d(k=12) == EINVAL and d(dst=a + 4) == EALIGN and d(n=0, c=None) == 0
    m = lambda xc=a, h=a, n=4, di=64, do=64: lib.molora_mx_matmul(xc, a, a, a, h, n, di, do, None)
    assert m(xc=None) == EINVAL and m(do=12) == EINVAL and m(di=0) == EINVAL and m(h=a + 8) == EALIGN and m(n=0, xc=None) == 0
    assert m(n=1 << 31) == EINVAL
    p = lambda x=a, r=a, n=4, rank=8, ws=a, nb=1 << 20: lib.molora_apply_mx(x, a, a, a, a, r, a, n, 64, 64, 2, rank, ws, nb, None)
    assert p(x=None) == EINVAL and p(r=None) == EINVAL and p(rank=12) == EINVAL and p(ws=None) == EINVAL
    assert p(ws=a + 16) == EALIGN and p(nb=64) == EWORKSPACE and p(r=a + 4) == EALIGN and p(n=0, x=None) == 0


def test_gated_entry_points_reject_bad_arguments(lib, a):
    def fwd(x=a, A=a, B=a, r=a, z=a, pre=None, n=4, di=64, F=32, C=2, rank=8, act=0, ws=a, nb=1 << 20):
        return lib.molora_apply_gated(x, a, A, B, r, z, pre, n, di, F, C, rank, act, ws, nb, None)
    assert fwd(x=None) == EINVAL and fwd(z=None) == EINVAL and fwd(act=3) == EINVAL and fwd(act=-1) == EINVAL
    assert fwd(F=12) == EINVAL and fwd(F=0) == EINVAL and fwd(rank=136) == EINVAL and fwd(di=60) == EINVAL
    assert fwd(A=None) == EINVAL and fwd(r=None) == EINVAL and fwd(C=0, rank=0) == EINVAL     # adapters given or not, not half
    assert fwd(A=None, B=None, r=None) == EINVAL and fwd(C=0, rank=8) == EINVAL and fwd(ws=None) == EINVAL
    assert fwd(z=a + 8) == EALIGN and fwd(pre=a + 8) == EALIGN and fwd(ws=a + 64) == EALIGN and fwd(nb=100) == EWORKSPACE
    assert fwd(n=0, x=None, z=None, ws=None) == 0
    assert fwd(n=1 << 20, di=2048) == EINVAL and fwd(di=65536, F=16384, n=100) == EINVAL      # 4 GiB of x, of W

    def bwd(dz=a, pre=a, dx=a, dA=a, dB=a, A=a, B=a, r=a, n=4, C=2, rank=8, act=0, ws=a, nb=1 << 24):
        return lib.molora_gated_backward(dz, a, a, A, B, r, pre, dx, a, dA, dB, n, 64, 32, C, rank, act, ws, nb, None)
    assert bwd(dz=None) == EINVAL and bwd(pre=None) == EINVAL and bwd(act=9) == EINVAL and bwd(ws=None) == EINVAL
    assert bwd(A=None) == EINVAL and bwd(A=None, B=None, r=None, C=0, rank=0) == EINVAL       # dA, dB of no adapters
    assert bwd(dx=a + 8) == EALIGN and bwd(dA=a + 2) == EALIGN and bwd(ws=a + 16) == EALIGN and bwd(nb=4096) == EWORKSPACE


# ---- refusals of the binding ----

def t(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


def test_binding_checks_come_before_the_device(lib):
    c, s = t(1, 1, 64, 16, dtype=u8), t(1, 1, 64, 4, dtype=u8)
    x, A, B, r = t(16, 64), t(2, 64, 8), t(2, 8, 32), t(16, dtype=i32)
    wc, ws = t(2, 1, 64, 16, dtype=u8), t(2, 1, 64, 4, dtype=u8)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        mb.molora_mx_quantize(t(16, 64, dtype=torch.float16))
    with pytest.raises(ValueError, match="2-D"):
        mb.molora_mx_quantize(t(16))
    with pytest.raises(ValueError, match="multiple of 8"):
        mb.molora_mx_quantize(t(16, 60))
    with pytest.raises(ValueError, match="x codes must have shape"):
        mb.molora_mx_quantize(t(17, 64), codes=c, scales=s)
    with pytest.raises(ValueError, match="contiguous"):
        mb.molora_mx_quantize(t(64, 16).t(), codes=c, scales=s)
    with pytest.raises(TypeError, match="device tensor"):
        mb.molora_mx_quantize(x, codes=c, scales=s)
    with pytest.raises(TypeError, match="W must be"):
        mb.molora_mx_quantize_w(t(64, 32, dtype=f32), codes=wc, scales=ws)
    with pytest.raises(ValueError, match="operand scales"):
        mb.molora_mx_dequantize(c, t(1, 2, 64, 4, dtype=u8), 16, 64)
    with pytest.raises(ValueError, match="W codes"):
        mb.molora_mx_matmul(c, s, c, s, 16, 64, 32)
    with pytest.raises(ValueError, match="h must have shape"):
        mb.molora_mx_matmul(c, s, wc, ws, 16, 64, 32, h=t(16, 40, dtype=f32))
    with pytest.raises(ValueError, match="B must have shape"):
        mb.molora_apply_mx(x, wc, ws, A, t(2, 16, 32), r)
    with pytest.raises(ValueError, match="r must have shape"):
        mb.molora_apply_mx(x, wc, ws, A, B, t(15, dtype=i32))
    with pytest.raises(TypeError, match="device tensor"):
        mb.molora_apply_mx(x, wc, ws, A, B, r)
    W = t(64, 32)
    with pytest.raises(ValueError, match="act must be"):
        mb.molora_apply_gated(x, W, act="relu")
    with pytest.raises(ValueError, match="given together"):
        mb.molora_apply_gated(x, W, A, B)
    with pytest.raises(ValueError, match="same width"):
        mb.molora_apply_gated(x, t(64, 31))
    with pytest.raises(ValueError, match="pre must have shape"):
        mb.molora_apply_gated(x, W, A, B, r, pre=t(16, 16, dtype=f32))
    with pytest.raises(ValueError, match="A must have shape"):
        mb.molora_apply_gated(x, W, t(2, 72, 8), B, r)
    with pytest.raises(TypeError, match="device tensor"):
        mb.molora_apply_gated(x, W, A, B, r)
    pre, dz = t(16, 32, dtype=f32), t(16, 16)
    with pytest.raises(ValueError, match="need names"):
        mb.molora_gated_backward(dz, x, W, A, B, r, pre, need=("x", "Q"))
    with pytest.raises(ValueError, match="dW is given"):
        mb.molora_gated_backward(dz, x, W, A, B, r, pre, need=("x",), dW=W)
    with pytest.raises(ValueError, match="dz must have shape"):
        mb.molora_gated_backward(t(16, 24), x, W, A, B, r, pre)
    with pytest.raises(TypeError, match="pre must be a tensor|pre must be"):
        mb.molora_gated_backward(dz, x, W, A, B, r, t(16, 32))
    with pytest.raises(TypeError, match="device tensor"):
        mb.molora_gated_backward(dz, x, W, A, B, r, pre)
