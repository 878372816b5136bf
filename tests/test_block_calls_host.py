"""Arguments of the feed-forward block's calls that the binding has to look at more closely, without a GPU."""
import pytest
import torch

from paper_2603_15965_amd import binding as mb

bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def t(*shape, dtype=bf):
    return torch.zeros(shape, dtype=dtype)


def test_need_may_be_any_iterable():
    """A generator is read once: dx is needed, so its buffer is taken (and then found to be on the host)."""
    x, W, A, B, r = t(16, 64), t(64, 32), t(2, 64, 8), t(2, 8, 32), t(16, dtype=i32)
    pre, dz = t(16, 32, dtype=f32), t(16, 16)
    for need in (("x",), ["x"], "x", iter(["x"]), (c for c in "x"), {"x": 1}):
        with pytest.raises(TypeError, match="device tensor"):
            mb.molora_gated_backward(dz, x, W, A, B, r, pre, need=need, dx=t(16, 64))
    with pytest.raises(ValueError, match="dx is given but not needed"):
        mb.molora_gated_backward(dz, x, W, A, B, r, pre, need=iter(["W"]), dx=t(16, 64))


@pytest.mark.parametrize("more", [8, 64])
def test_sizes_that_do_not_fit_32_bits_are_refused(more):
    """2^32 + 8 columns are not 8: what the library would be told is looked at before anything is allocated."""
    wide = (1 << 32) + more
    with pytest.raises(ValueError, match="2\\^31"):
        mb.molora_mx_quantize(torch.empty(1, wide, dtype=bf, device="meta"))
    with pytest.raises(ValueError, match="2\\^31"):
        mb.molora_mx_quantize_w(torch.empty(8, wide, dtype=bf, device="meta"))
    with pytest.raises(ValueError, match="2\\^31"):
        mb.molora_mx_dequantize(t(1, 1, 64, 16, dtype=u8), t(1, 1, 64, 4, dtype=u8), 1, wide)
    with pytest.raises(ValueError, match="2\\^31"):
        mb.molora_apply_gated(t(1, 8), torch.empty(8, 2 * wide, dtype=bf, device="meta"))


def test_gradients_of_adapters_beyond_a_launch_are_refused_at_once():
    """Sizes whose last launches do not fit a grid: refused with the others, not when the first ones are on their way."""
    import ctypes
    lib = mb.load()
    buf = (ctypes.c_char * 512)()
    a = ctypes.addressof(buf)
    a += -a % 256

    def call(N, d_in, F, C, rank):
        ws = lib.molora_gated_backward_workspace_bytes(N, d_in, F, C, rank)
        return ws, lib.molora_gated_backward(a, a, a, a, a, a, a, a, a, a, a, N, d_in, F, C, rank, 0, a, 1 << 40, None)
    for sizes in ((2000, 8, 1 << 19, 1024, 8), (500, 8, 1 << 21, 1024, 8), (16, 1 << 20, 1016, 1024, 16)):
        assert call(*sizes) == (0, -1), sizes
    assert lib.molora_gated_backward_workspace_bytes(2000, 8, 1 << 18, 1024, 8) > 0
    assert lib.molora_gated_backward_workspace_bytes(8000, 8, 1 << 16, 1024, 128) > 0
    assert lib.molora_apply_gated_workspace_bytes(2000, 8, 1 << 19, 1024, 8) > 0   # the forward pass has no such launch
