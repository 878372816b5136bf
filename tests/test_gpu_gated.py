"""The gated block and its backward pass on the GPU against the 64-bit definition, and the block as it is used:
gated projection, down projection on a 4-bit weight, captured and replayed."""
import numpy as np
import pytest

import block_reference as ref
from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu
ACTS = ["silu", "gelu", "gelu_tanh"]


def _gpu():
    import torch
    from paper_2603_15965_amd import binding as mb
    return torch, mb


def _case(N, d_in, F, C, rank, how="mixed", seed=0):
    w = wl.custom("gated", N, d_in, 2 * F, max(C, 1), rank if C else 8, 5000 + seed + 31 * N + d_in + wl.BASE_SEED)
    rng = np.random.default_rng(N + F)
    r = rng.integers(0, max(C, 1), N).astype(np.int32)
    if how == "mixed":
        r[::6], r[4::9] = -1, C + 1
    elif how == "none":
        r[:] = -1
    elif how == "last":
        r[:] = C - 1
    elif how == "ends":   # two long buckets, short and empty ones between them
        r[:N * 3 // 10], r[N * 4 // 10:] = 0, C - 1
    dz = wl.to_bf16_bits(rng.standard_normal((N, F)).astype(np.float32))
    return w, r, dz


def _tensors(torch, mb, w, r, C):
    x, W = mb.bf16_tensor(w.x), mb.bf16_tensor(w.W)
    return (x, W, mb.bf16_tensor(w.A), mb.bf16_tensor(w.B), torch.from_numpy(r).cuda()) if C else (x, W, None, None, None)


def _numbers(w, r, C):
    return (ref.f64(w.x), ref.f64(w.W)) + ((ref.f64(w.A), ref.f64(w.B), r) if C else (None, None, None))


def _guarded(torch, shape, dtype, fill=7.0):
    n = int(np.prod(shape))
    room = torch.full((n + 512,), fill, dtype=dtype, device="cuda")
    return room[256:256 + n].view(shape), lambda: bool((room[:256] == fill).all() and (room[256 + n:] == fill).all())


FORWARD = [(1, 64, 8, 1, 8, "last"), (1, 512, 264, 4, 16, "mixed"), (7, 136, 40, 3, 16, "mixed"), (33, 264, 72, 5, 24, "mixed"),
           (64, 256, 136, 6, 64, "mixed"), (64, 128, 24, 3, 128, "none"), (65, 64, 8, 1, 8, "last"), (66, 136, 40, 3, 16, "mixed"),
           (130, 264, 200, 5, 40, "mixed"), (300, 520, 264, 64, 16, "mixed"), (515, 1032, 328, 7, 24, "mixed"), (600, 72, 520, 2, 128, "mixed"),
           (5, 2056, 8328, 3, 16, "mixed"), (1, 64, 24, 0, 0, "none"), (40, 264, 136, 0, 0, "none"), (200, 136, 264, 0, 0, "none")]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("N,d_in,F,C,rank,how", FORWARD)
def test_forward_matches_the_definition(N, d_in, F, C, rank, how, act):
    torch, mb = _gpu()
    print(f"gated {act} {N} x {d_in} -> 2 x {F}, {C} of rank {rank}, {how}", flush=True)
    w, r, _ = _case(N, d_in, F, C, rank, how)
    args = _tensors(torch, mb, w, r, C)
    z, z_ok = _guarded(torch, (N, F), torch.bfloat16)
    pre, p_ok = _guarded(torch, (N, 2 * F), torch.float32)
    mb.molora_apply_gated(*args, act=act, z=z, pre=pre)
    torch.cuda.synchronize()
    assert z_ok() and p_ok()
    h, off = ref.projection(*_numbers(w, r, C))
    assert (np.abs(pre.cpu().numpy() - h) <= off).all()
    want = ref.act(h[:, :F], act)[0] * h[:, F:]
    assert (np.abs(z.float().cpu().numpy() - want) <= ref.gated_off(h, off, act)).all()
    assert torch.equal(z, mb.molora_apply_gated(*args, act=act)), "without pre: other bits"


BACKWARD = [(1, 64, 8, 1, 8, "last"), (1, 64, 8, 2, 8, "none"), (7, 136, 40, 3, 16, "mixed"), (64, 256, 136, 6, 64, "mixed"),
            (65, 72, 24, 2, 128, "mixed"), (130, 264, 200, 5, 40, "mixed"), (515, 520, 264, 7, 24, "mixed"), (300, 128, 136, 40, 16, "mixed"),
            (33, 136, 72, 0, 0, "none"), (200, 264, 136, 0, 0, "none"), (257, 64, 64, 3, 8, "none"),
            # few output tiles: K in slices (of dx: 2 F, of dW: the tokens), rows of a bucket in pieces, the last ones ragged
            (96, 72, 1040, 2, 16, "mixed"), (2056, 64, 40, 2, 16, "mixed"), (3001, 136, 72, 1, 40, "last"), (1500, 64, 1032, 0, 0, "none"),
            (4100, 72, 40, 70, 24, "last"), (5003, 64, 72, 131, 8, "ends"),
            (515, 520, 264, 70, 40, "mixed"), (4100, 136, 584, 67, 40, "ends")]   # wavefronts by columns


@pytest.mark.parametrize("N,d_in,F,C,rank,how,act", [c + (ACTS[i % 3],) for i, c in enumerate(BACKWARD)])
def test_backward_matches_the_definition(N, d_in, F, C, rank, how, act):
    torch, mb = _gpu()
    print(f"gated backward {act} {N} x {d_in} -> 2 x {F}, {C} of rank {rank}, {how}", flush=True)
    w, r, dzb = _case(N, d_in, F, C, rank, how)
    args = _tensors(torch, mb, w, r, C)
    dz, pre = mb.bf16_tensor(dzb), torch.empty(N, 2 * F, dtype=torch.float32, device="cuda")
    mb.molora_apply_gated(*args, act=act, pre=pre)
    nbytes = int(mb.load().molora_gated_backward_workspace_bytes(N, d_in, F, C, rank))
    room = torch.full((nbytes + 512,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN wherever it is read unwritten
    shapes = {"dx": (N, d_in), "dW": (d_in, 2 * F)} | ({"dA": (C, d_in, rank), "dB": (C, rank, 2 * F)} if C else {})
    bufs = {k: _guarded(torch, s, torch.bfloat16) for k, s in shapes.items()}
    got = mb.molora_gated_backward(dz, *args, pre, act=act, workspace=room[256:256 + nbytes], **{k: b[0] for k, b in bufs.items()})
    torch.cuda.synchronize()
    assert bool((room[:256] == 0xFF).all() and (room[256 + nbytes:] == 0xFF).all())
    want = ref.gated_gradients(ref.f64(dzb), *_numbers(w, r, C), act)
    for i, k in enumerate(("dx", "dW", "dA", "dB")):
        if k not in want:
            assert got[i] is None
            continue
        v, off = want[k]
        g = got[i].double().cpu().numpy()
        assert bufs[k][1](), f"{k}: written beyond its end"
        assert (np.abs(g - v) <= off).all(), f"{k}: {np.max(np.abs(g - v) / np.maximum(off, 1e-300))} of the bound"
        # two roundings to bf16, each off by at most 2^-8 / sqrt(3) in the mean square: 0.82 of this together
        if v.any():
            assert np.linalg.norm(g - v) <= ref.HALF16 * np.linalg.norm(v), k
    # each gradient by itself: the same bits
    for i, k in enumerate("xWAB" if C else "xW"):
        alone = mb.molora_gated_backward(dz, *args, pre, act=act, need=(k,))
        assert torch.equal(alone[i], got[i]), f"d{k} alone"
        assert all(t is None for j, t in enumerate(alone) if j != i)


def test_no_tokens():
    torch, mb = _gpu()
    w, r, dzb = _case(8, 64, 16, 3, 8)
    x, W, A, B, rr = _tensors(torch, mb, w, r, 3)
    e = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
    z = mb.molora_apply_gated(x[:0], W, A, B, rr[:0])
    assert z.shape == (0, 16)
    dx, dW, dA, dB = mb.molora_gated_backward(e(0, 16), x[:0], W, A, B, rr[:0], e(0, 32, dtype=torch.float32))
    assert dx.shape == (0, 64) and not dW.any() and not dA.any() and not dB.any()
    wc, ws = mb.molora_mx_quantize_w(W)
    assert mb.molora_apply_mx(x[:0], wc, ws, A, B, rr[:0]).shape == (0, 32)
    xc, xs = mb.molora_mx_quantize(x[:0])
    assert mb.molora_mx_matmul(xc, xs, wc, ws, 0, 64, 32).shape == (0, 32)


@pytest.mark.parametrize("act", ACTS)
def test_far_values(act):
    """Gates of +-1 .. +-1e4: act and its slope go to their limits, nothing overflows to NaN."""
    torch, mb = _gpu()
    N, F = 64, 16
    pre = torch.zeros(N, 2 * F, dtype=torch.float32, device="cuda")
    g = torch.logspace(0, 4, N * F // 2, device="cuda")
    pre[:, :F] = torch.cat((g, -g)).view(N, F)
    pre[:, F:] = 1.5
    dz = torch.ones(N, F, dtype=torch.bfloat16, device="cuda")
    x = torch.eye(64, dtype=torch.bfloat16, device="cuda")
    W = torch.zeros(64, 2 * F, dtype=torch.bfloat16, device="cuda")
    dW = mb.molora_gated_backward(dz, x, W, None, None, None, pre, act=act, need=("W",))[1]   # x = 1: dW = dh
    h = pre.double().cpu().numpy()
    a, da = ref.act(h[:, :F], act)
    want = np.concatenate((1.5 * da, a), 1)
    # fp32 evaluation: the exponent's argument is off by steps of itself, up to |g|^3
    off = 2 * ref.HALF16 * np.abs(want) + 1e-6
    assert np.isfinite(dW.float().cpu().numpy()).all()
    assert (np.abs(dW.double().cpu().numpy() - want) <= off).all()


@pytest.mark.parametrize("N", [48, 200])
def test_block_in_a_graph_and_on_another_stream(N):
    """Gated projection, its gradients, and the down projection on a 4-bit weight: captured once, replayed with
    inputs renewed in place and eager work between, against the eager calls on the default stream."""
    torch, mb = _gpu()
    d, F, C, rank = 264, 136, 4, 16
    w, r, dzb = _case(N, d, F, C, rank)
    x, W, A, B, rr = _tensors(torch, mb, w, r, C)
    down = wl.custom("down", N, F, d, C, rank, 41 + wl.BASE_SEED)
    A2, B2 = mb.bf16_tensor(down.A), mb.bf16_tensor(down.B)
    wc, ws = mb.molora_mx_quantize_w(mb.bf16_tensor(down.W))
    dz = mb.bf16_tensor(dzb)
    lib = mb.load()
    room = lambda fn, *sizes: torch.empty(max(256, getattr(lib, fn)(*sizes)), dtype=torch.uint8, device="cuda")

    def buffers():
        e = lambda *s, dtype=torch.bfloat16: torch.full(s, 3.0, dtype=dtype, device="cuda")
        return dict(z=e(N, F), pre=e(N, 2 * F, dtype=torch.float32), y=e(N, d, dtype=torch.float32), dx=e(N, d), dW=e(d, 2 * F),
                    dA=e(C, d, rank), dB=e(C, rank, 2 * F), w1=room("molora_apply_gated_workspace_bytes", N, d, F, C, rank),
                    w2=room("molora_apply_mx_workspace_bytes", N, F, d, C, rank),
                    w3=room("molora_gated_backward_workspace_bytes", N, d, F, C, rank))

    def block(b, stream=None):
        mb.molora_apply_gated(x, W, A, B, rr, z=b["z"], pre=b["pre"], workspace=b["w1"], stream=stream)
        mb.molora_apply_mx(b["z"], wc, ws, A2, B2, rr, h=b["y"], workspace=b["w2"], stream=stream)
        mb.molora_gated_backward(dz, x, W, A, B, rr, b["pre"], dx=b["dx"], dW=b["dW"], dA=b["dA"], dB=b["dB"], workspace=b["w3"],
                                 stream=stream)

    side = torch.cuda.Stream()
    mine, two = buffers(), buffers()
    torch.cuda.synchronize()
    graphs = []
    for b in (mine, two):     # two graphs, each with workspaces of its own
        g = mb.Graph(side)
        with g.capture():
            block(b, side)
        graphs.append((g, b))
    rng = np.random.default_rng(2)
    for replay in range(4):
        if replay:
            x.copy_(mb.bf16_tensor(w.x[rng.permutation(N)]))
            rr.copy_(torch.from_numpy(r[rng.permutation(N)]).cuda())
        eager = buffers()
        block(eager)
        torch.cuda.synchronize()
        for g, b in graphs:
            g.launch()
        side.synchronize()
        for _, b in graphs:
            for k in ("z", "pre", "y", "dx", "dW", "dA", "dB"):
                assert torch.equal(b[k], eager[k]), f"replay {replay}: {k}"
    for g, _ in graphs:
        g.destroy()
    # the down projection takes what the gated one gave
    want = ref.mx_values(mine["z"].double().cpu().numpy()) @ ref.mx_values(ref.f64(down.W).T).T
    l, _ = ref.lora(mine["z"].double().cpu().numpy(), ref.f64(down.A), ref.f64(down.B), rr.cpu().numpy())
    y = mine["y"].cpu().numpy()
    assert np.linalg.norm(y - want - l) <= (F * ref.ULP32 + ref.HALF16 ** 2) * np.linalg.norm(np.abs(want) + np.abs(l)) * 4


def test_tensors_of_another_device_are_refused(monkeypatch):
    torch, mb = _gpu()
    w, r, dzb = _case(8, 64, 16, 3, 8)
    args = _tensors(torch, mb, w, r, 3)
    z = torch.full((8, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    wc, ws = mb.molora_mx_quantize_w(args[1])
    monkeypatch.setattr(mb, "_raw_device", lambda: 1)
    with pytest.raises(ValueError, match="the current device is cuda:1"):
        mb.molora_apply_gated(*args, z=z)
    with pytest.raises(ValueError, match="the current device is cuda:1"):
        mb.molora_apply_mx(args[0], wc, ws, *args[2:])
    with pytest.raises(ValueError, match="the current device is cuda:1"):
        mb.molora_mx_quantize(args[0])
    assert bool((z == 7).all())


def test_another_stream_and_workspaces_of_the_calls_own():
    """Calls on a side stream that allocate their workspaces, while the default stream allocates and fills memory of
    the same size: nothing of what the side stream still uses may be handed out."""
    torch, mb = _gpu()
    N, d, F, C, rank = 300, 264, 520, 4, 16
    w, r, dzb = _case(N, d, F, C, rank)
    args = _tensors(torch, mb, w, r, C)
    dz = mb.bf16_tensor(dzb)
    wc, ws = mb.molora_mx_quantize_w(args[1])
    pre = torch.empty(N, 2 * F, dtype=torch.float32, device="cuda")
    z = mb.molora_apply_gated(*args, pre=pre)
    want = (z, *mb.molora_gated_backward(dz, *args, pre), mb.molora_apply_mx(args[0], wc, ws, *args[2:]))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    sizes = [int(f(N, d, F, C, rank)) for f in (mb.load().molora_apply_gated_workspace_bytes, mb.load().molora_gated_backward_workspace_bytes)]
    for handle in (side, side.cuda_stream):
        for _ in range(3):
            outs = [torch.empty_like(t) for t in want]
            torch.cuda.synchronize()
            mb.molora_apply_gated(*args, z=outs[0], stream=handle)
            mb.molora_gated_backward(dz, *args, pre, dx=outs[1], dW=outs[2], dA=outs[3], dB=outs[4], stream=handle)
            mb.molora_apply_mx(args[0], wc, ws, *args[2:], h=outs[5], stream=handle)
            for n in sizes:
                torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))
