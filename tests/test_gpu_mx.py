"""4-bit microscaled operands and their products on the GPU against the 64-bit definition: codes bit for bit,
sums within what fp32 additions can be off by."""
import numpy as np
import pytest

import block_reference as ref
from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _gpu():
    import torch
    from paper_2603_15965_amd import binding as mb
    return torch, mb


def _bits(shape, seed, std=1.0):
    return wl.normal_bf16(seed, shape, std)


def _guarded(torch, shape, dtype, fill):
    """A tensor inside a larger one, and a check that what lies around it is untouched."""
    n = int(np.prod(shape))
    room = torch.full((n + 512,), fill, dtype=dtype, device="cuda")
    return room[256:256 + n].view(shape), lambda: bool((room[:256] == fill).all() and (room[256 + n:] == fill).all())


def _quantize(torch, mb, v, weight=False):
    rows, K = (v.shape[1], v.shape[0]) if weight else v.shape
    c, s = mb._mx_shapes(rows, K)
    codes, c_ok = _guarded(torch, c, torch.uint8, 0xA5)
    scales, s_ok = _guarded(torch, s, torch.uint8, 0xA5)
    (mb.molora_mx_quantize_w if weight else mb.molora_mx_quantize)(v, codes, scales)
    torch.cuda.synchronize()
    assert c_ok() and s_ok()
    return codes, scales


def _same_blocks(torch, codes, scales, v, what):
    """Equal to the definition's: scales always, codes but where the block is NaN."""
    q, s = ref.mx_packed(v)
    gq, gs = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.array_equal(gs, s), f"{what}: {np.sum(gs != s)} scales differ"
    nan = (s == 255).transpose(0, 1, 3, 2).reshape(s.shape[0], -1, 64)[:, :q.shape[1]]
    diff = (gq != q).any(-1) & ~nan
    assert not diff.any(), f"{what}: codes of {diff.sum()} blocks differ, first {np.argwhere(diff)[0]}"


@pytest.mark.parametrize("rows,K", [(1, 8), (1, 128), (3, 40), (16, 512), (17, 520), (33, 136), (515, 1032), (64, 2728)])
@pytest.mark.parametrize("kind", ["bf16", "fp32", "weight"])
def test_quantize_matches_the_definition(rows, K, kind):
    torch, mb = _gpu()
    print(f"quantize {kind} {rows} x {K}", flush=True)
    if kind == "weight":
        rows = (rows + 7) // 8 * 8
        bits = _bits((K, rows), rows + K)
        codes, scales = _quantize(torch, mb, mb.bf16_tensor(bits), weight=True)
        v = ref.f64(bits).T
    elif kind == "bf16":
        bits = _bits((rows, K), rows + K, 3.0)
        codes, scales = _quantize(torch, mb, mb.bf16_tensor(bits))
        v = ref.f64(bits)
    else:
        v = np.random.default_rng(rows + K).standard_normal((rows, K)).astype(np.float32)
        codes, scales = _quantize(torch, mb, torch.from_numpy(v).cuda())
    _same_blocks(torch, codes, scales, np.asarray(v, np.float64), kind)
    rows = v.shape[0]
    out, ok = _guarded(torch, (rows, K), torch.float32, 7.0)
    mb.molora_mx_dequantize(codes, scales, rows, K, out)
    torch.cuda.synchronize()
    assert ok() and np.array_equal(out.cpu().numpy().astype(np.float64), ref.mx_values(np.asarray(v, np.float64)))


@pytest.mark.parametrize("top", [0x0001, 0x007F, 0x0080, 0x0100, 0x0180, 0x3F80, 0x3FFF, 0x4049, 0x7F00, 0x7F7F])
def test_quantize_every_bf16_value_under_a_maximum(top):
    """Every bf16 number up to the block's maximum, both signs, from the subnormal ones to the largest."""
    torch, mb = _gpu()
    print(f"quantize all values up to {top:#06x}", flush=True)
    vals = np.arange(0, top + 1, dtype=np.uint16)
    vals = np.concatenate((vals, vals | 0x8000))
    vals = np.pad(vals, (0, -len(vals) % 31)).reshape(-1, 31)
    bits = np.concatenate((np.full((len(vals), 1), top, np.uint16), vals), 1)
    bits = np.pad(bits, ((0, -len(bits) % 8), (0, 0)))
    for weight in (False, True):
        v = mb.bf16_tensor(np.ascontiguousarray(bits.T) if weight else bits)
        codes, scales = _quantize(torch, mb, v, weight)
        _same_blocks(torch, codes, scales, ref.f64(bits), f"weight {weight}")
    out = mb.molora_mx_dequantize(codes, scales, len(bits), 32).cpu().numpy().astype(np.float64)
    assert np.array_equal(out, ref.mx_values(ref.f64(bits)))


def test_quantize_fp32_borders():
    """fp32 numbers a step below, on and above every border between codes, at many powers of two."""
    torch, mb = _gpu()
    mids = np.array([.25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7.9999], np.float32)
    near = np.concatenate((np.nextafter(mids, np.float32(0)), mids, np.nextafter(mids, np.float32(9))))
    near = np.concatenate((near, [4.0, 0, 0, 0, 0])).astype(np.float32)
    v = np.stack([near * s * np.float32(2.0) ** e for e in (-126, -124, -100, -24, -1, 0, 1, 30, 100, 124) for s in (1, -1)])
    codes, scales = _quantize(torch, mb, torch.from_numpy(v.astype(np.float32)).cuda())
    _same_blocks(torch, codes, scales, v.astype(np.float64), "borders")


def test_blocks_that_are_not_finite_stand_for_nan_and_no_other_does():
    torch, mb = _gpu()
    bits = _bits((40, 264), 3)
    bits[3, 40], bits[3, 100], bits[20, 263], bits[39, 0] = 0x7F80, 0x7FC0, 0xFF80, 0xFFFF
    for weight in (False, True):
        v = mb.bf16_tensor(np.ascontiguousarray(bits.T) if weight else bits)
        codes, scales = _quantize(torch, mb, v, weight)
        _same_blocks(torch, codes, scales, ref.f64(bits), f"weight {weight}")
        got = mb.molora_mx_dequantize(codes, scales, 40, 264).cpu().numpy()
        nan = np.zeros((40, 264), bool)
        nan[3, 32:64] = nan[3, 96:128] = nan[20, 256:] = nan[39, :32] = True
        assert np.array_equal(np.isnan(got), nan)
    # a row of the product with such a block is NaN, the other rows are what they were
    W = mb.bf16_tensor(_bits((264, 48), 4))
    wc, ws = mb.molora_mx_quantize_w(W)
    xc, xs = mb.molora_mx_quantize(mb.bf16_tensor(bits))
    h = mb.molora_mx_matmul(xc, xs, wc, ws, 40, 264, 48).cpu().numpy()
    bad = np.zeros(40, bool)
    bad[[3, 20, 39]] = True
    assert np.array_equal(np.isnan(h).all(1), bad) and np.array_equal(np.isnan(h).any(1), bad)


def _product_ref(xb, Wb):
    qx, qw = ref.mx_values(ref.f64(xb)), ref.mx_values(ref.f64(Wb).T)
    return qx @ qw.T, (xb.shape[1] + 1) * ref.ULP32 * (np.abs(qx) @ np.abs(qw).T)


@pytest.mark.parametrize("N", [1, 2, 16, 17, 33, 48, 63, 64, 65, 127, 128, 300])
@pytest.mark.parametrize("d_in,d_out", [(8, 8), (40, 264), (128, 24), (136, 16), (520, 72), (1032, 392), (2048, 128)])
def test_matmul_matches_the_definition(N, d_in, d_out):
    torch, mb = _gpu()
    print(f"matmul {N} x {d_in} -> {d_out}", flush=True)
    xb, Wb = _bits((N, d_in), N + d_in), _bits((d_in, d_out), d_out, d_in ** -0.5)
    xb[:, d_in // 2] = _bits((N,), 9, 30.0)      # blocks of very different scales
    wc, ws = mb.molora_mx_quantize_w(mb.bf16_tensor(Wb))
    xc, xs = mb.molora_mx_quantize(mb.bf16_tensor(xb))
    h, ok = _guarded(torch, (N, d_out), torch.float32, 7.0)
    mb.molora_mx_matmul(xc, xs, wc, ws, N, d_in, d_out, h)
    torch.cuda.synchronize()
    want, off = _product_ref(xb, Wb)
    assert ok() and (np.abs(h.cpu().numpy() - want) <= off).all()
    again = mb.molora_mx_matmul(xc, xs, wc, ws, N, d_in, d_out)
    assert torch.equal(h, again)


@pytest.mark.parametrize("N,d_in,d_out", [(4096, 264, 4104), (2050, 1032, 9000), (70, 12288, 520), (64, 12288, 40)])
def test_matmul_large(N, d_in, d_out):
    """Sizes of the large tiles and of long sums, against 64-bit products on the device."""
    torch, mb = _gpu()
    print(f"matmul large {N} x {d_in} -> {d_out}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randn(N, d_in, generator=g, device="cuda").bfloat16()
    W = (torch.randn(d_in, d_out, generator=g, device="cuda") * d_in ** -0.5).bfloat16()
    wc, ws = mb.molora_mx_quantize_w(W)
    xc, xs = mb.molora_mx_quantize(x)
    qx = mb.molora_mx_dequantize(xc, xs, N, d_in).double()
    qw = mb.molora_mx_dequantize(wc, ws, d_out, d_in).double()
    rows = np.random.default_rng(1).choice(N, min(N, 64), replace=False)
    assert np.array_equal(qx[rows].cpu().numpy(), ref.mx_values(x[rows].double().cpu().numpy()))
    h = mb.molora_mx_matmul(xc, xs, wc, ws, N, d_in, d_out)
    want, off = qx @ qw.t().contiguous(), (d_in + 1) * ref.ULP32 * (qx.abs() @ qw.abs().t().contiguous())
    assert bool(((h.double() - want).abs() <= off).all())


def _targets(N, C, seed, how):
    rng = np.random.default_rng(seed)
    if how == "none":
        return np.full(N, -1, np.int32)
    if how == "one":
        return np.full(N, C - 1, np.int32)
    r = rng.integers(0, C, N).astype(np.int32)
    r[::7], r[3::11] = -1, C + 3
    return r


APPLY = [(1, 64, 8, 1, 8, "one"), (5, 136, 40, 3, 16, "mixed"), (16, 264, 264, 4, 24, "mixed"), (64, 520, 128, 6, 64, "mixed"),
         (63, 256, 72, 40, 128, "mixed"), (64, 256, 72, 4, 8, "none"), (65, 128, 136, 3, 8, "mixed"), (130, 264, 392, 5, 40, "mixed"),
         (300, 520, 264, 64, 16, "mixed"), (257, 136, 8, 2, 128, "one"), (515, 1032, 520, 7, 24, "mixed"), (200, 128, 128, 4, 16, "none")]


@pytest.mark.parametrize("N,d_in,d_out,C,rank,how", APPLY)
def test_apply_mx_matches_the_definition(N, d_in, d_out, C, rank, how):
    torch, mb = _gpu()
    print(f"apply_mx {N} x {d_in} -> {d_out}, {C} of rank {rank}, {how}", flush=True)
    w = wl.custom("mx", N, d_in, d_out, C, rank, 900 + N + wl.BASE_SEED)
    r = _targets(N, C, N, how)
    x, A, B = (mb.bf16_tensor(t) for t in (w.x, w.A, w.B))
    wc, ws = mb.molora_mx_quantize_w(mb.bf16_tensor(w.W))
    h, ok = _guarded(torch, (N, d_out), torch.float32, 7.0)
    nbytes = int(mb.load().molora_apply_mx_workspace_bytes(N, d_in, d_out, C, rank))
    room = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    mb.molora_apply_mx(x, wc, ws, A, B, torch.from_numpy(r).cuda(), h, workspace=room[256:256 + nbytes])
    torch.cuda.synchronize()
    want, off = _product_ref(w.x, w.W)
    l, lo = ref.lora(ref.f64(w.x), ref.f64(w.A), ref.f64(w.B), r)
    assert ok() and bool((room[:256] == 0xA5).all() and (room[256 + nbytes:] == 0xA5).all())
    off = off + lo + 2 * ref.ULP32 * (np.abs(l) + np.abs(want))
    assert (np.abs(h.cpu().numpy() - want - l) <= off).all()


def test_apply_mx_many_buckets_in_large_tiles():
    """256-row tiles crossed by many small buckets, some rows without adapter."""
    torch, mb = _gpu()
    N, d_in, d_out, C, rank = 4100, 256, 4096, 100, 16
    w = wl.custom("mx", N, d_in, d_out, C, rank, 77 + wl.BASE_SEED, structure="zipf")
    r = w.r.copy()
    r[::5] = -1
    x, A, B = (mb.bf16_tensor(t) for t in (w.x, w.A, w.B))
    wc, ws = mb.molora_mx_quantize_w(mb.bf16_tensor(w.W))
    h = mb.molora_apply_mx(x, wc, ws, A, B, torch.from_numpy(r).cuda()).cpu().numpy()
    want, off = _product_ref(w.x, w.W)
    l, lo = ref.lora(ref.f64(w.x), ref.f64(w.A), ref.f64(w.B), r)
    assert (np.abs(h - want - l) <= off + lo + 2 * ref.ULP32 * (np.abs(l) + np.abs(want))).all()


def test_offsets_beyond_32_bits():
    """x of more than 4 GiB: the last rows as by themselves (codes the same, sums in another order)."""
    torch, mb = _gpu()
    N, d_in, d_out, C, rank, tail = 266256, 8200, 40, 3, 8, 112
    print(f"x {N} x {d_in}, {N * d_in * 2 / 2 ** 30:.2f} GiB", flush=True)
    torch.manual_seed(11)
    x = torch.empty(N, d_in, dtype=torch.bfloat16, device="cuda")
    for lo in range(0, N, 32768):
        x[lo:lo + 32768].normal_()
    W = (torch.randn(d_in, d_out, device="cuda") / d_in ** 0.5).bfloat16()
    A = (torch.randn(C, d_in, rank, device="cuda") / d_in ** 0.5).bfloat16()
    B = (torch.randn(C, rank, d_out, device="cuda") / rank ** 0.5).bfloat16()
    r = (torch.arange(N, device="cuda") % (C + 1)).to(torch.int32)   # one in four without adapter
    wc, ws = mb.molora_mx_quantize_w(W)
    assert N % 16 == 0 and tail % 16 == 0
    codes, scales = mb.molora_mx_quantize(x)
    c2, s2 = mb.molora_mx_quantize(x[-tail:])
    assert torch.equal(codes[-tail // 16:], c2) and torch.equal(scales[-tail // 16:], s2)
    h = mb.molora_mx_matmul(codes, scales, wc, ws, N, d_in, d_out)[-tail:]
    one = mb.molora_mx_matmul(c2, s2, wc, ws, tail, d_in, d_out)
    qx, qw = mb.molora_mx_dequantize(c2, s2, tail, d_in).abs().double(), mb.molora_mx_dequantize(wc, ws, d_out, d_in).abs().double()
    # two fp32 sums of d_in terms, each addition off by half a step
    off = 2 * d_in * 2.0 ** -24 * (qx @ qw.t().contiguous())
    assert bool(((h.double() - one.double()).abs() <= off).all())
    del codes, scales
    h = mb.molora_apply_mx(x, wc, ws, A, B, r)[-tail:]
    one = mb.molora_apply_mx(x[-tail:], wc, ws, A, B, r[-tail:])
    low = torch.zeros(tail, d_out, dtype=torch.float64, device="cuda")
    for c in range(C):
        mine = r[-tail:] == c
        low[mine] = x[-tail:][mine].double().abs() @ A[c].double().abs() @ B[c].double().abs()
    # t is a sum of d_in terms, carried as two bf16 halves (2^-17 together); then rank terms beside the others
    off += (2 * (d_in + 2 * rank) * 2.0 ** -24 + 2.0 ** -16) * low + 2 * 2 * rank * 2.0 ** -24 * (qx @ qw.t().contiguous())
    assert bool(((h.double() - one.double()).abs() <= off).all())
