"""The 4-bit projection of at most 64 tokens where few tokens have an adapter: which ones is asked of all lanes of a
wavefront, whatever row a lane itself works on."""
import numpy as np
import pytest

import block_reference as ref
from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 3, 9, 17, 31, 33, 47, 64])
@pytest.mark.parametrize("rank", [8, 40, 64, 128])
@pytest.mark.parametrize("who", ["last", "all but the first", "every third"])
def test_few_tokens_with_an_adapter(N, rank, who):
    import torch
    from paper_2603_15965_amd import binding as mb
    print(f"apply_mx {N} tokens, rank {rank}, adapters: {who}", flush=True)
    d_in, d_out, C = 136, 72, 3
    w = wl.custom("few", N, d_in, d_out, C, rank, wl.BASE_SEED + 62000 + N + rank)
    at = np.arange(N)
    has = {"last": at == N - 1, "all but the first": at > 0, "every third": at % 3 == 1}[who]
    r = np.where(has, at % C, -1).astype(np.int32)
    x, W, A, B = (mb.bf16_tensor(t) for t in (w.x, w.W, w.A, w.B))
    wc, ws = mb.molora_mx_quantize_w(W)
    nbytes = int(mb.load().molora_apply_mx_workspace_bytes(N, d_in, d_out, C, rank))
    work = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")   # NaN wherever it is read unwritten
    h = mb.molora_apply_mx(x, wc, ws, A, B, torch.from_numpy(r).cuda(), workspace=work).cpu().numpy()
    qx, qw = ref.mx_values(ref.f64(w.x)), ref.mx_values(ref.f64(w.W).T)
    want, off = qx @ qw.T, (d_in + 1) * ref.ULP32 * (np.abs(qx) @ np.abs(qw).T)
    l, lo = ref.lora(ref.f64(w.x), ref.f64(w.A), ref.f64(w.B), r)
    assert (np.abs(h - want - l) <= off + lo + 2 * ref.ULP32 * (np.abs(l) + np.abs(want))).all()
