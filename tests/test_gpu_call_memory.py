"""Memory that the calls of the routed projection allocate by themselves when they run on a stream other than the current
one, or are recorded."""
import numpy as np
import pytest

from paper_2603_15965_amd import workloads as wl

pytestmark = pytest.mark.gpu
N, D, DO, C, RANK, SMALL = 600, 264, 512, 4, 16, 48


def _calls():
    import torch
    from paper_2603_15965_amd import binding as mb
    w = wl.custom("memory", N, D, DO, C, RANK, 7300 + wl.BASE_SEED, route="gate")
    x, W, A, B, G = (mb.bf16_tensor(t) for t in (w.x, w.W, w.A, w.B, w.G))
    wide = wl.custom("memory", SMALL, D, DO, C, 64, 7301 + wl.BASE_SEED)
    xs, As, Bs = (mb.bf16_tensor(t) for t in (wide.x, wide.A, wide.B))
    rs = torch.from_numpy(wide.r).cuda()
    r = mb.molora_route(x, G)
    offsets, perm = mb.molora_bucket(r, C)
    t = mb.molora_shrink(x, A, offsets, perm)
    _, _, td = mb.molora_bucket_shrink(r, x, A)
    v = torch.from_numpy(np.random.default_rng(3).integers(0, 100, N).astype(np.int32)).cuda()
    ad = torch.from_numpy(np.random.default_rng(4).integers(0, 2, N).astype(np.int32)).cuda()
    breaks = [0, 50, 100]
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")
    W1, W2, b1, b2 = rn(D, 64).bfloat16(), rn(64, C).bfloat16(), rn(64), rn(C)
    idx = torch.stack((r, (r + 1) % C), 1).contiguous()
    torch.cuda.synchronize()
    one = lambda f: lambda s: (f(s),)
    return {
        "route": one(lambda s: mb.molora_route(x, G, stream=s)),
        "route_vocab": one(lambda s: mb.molora_route_vocab(v, breaks, stream=s)),
        "route_compose": one(lambda s: mb.molora_route_compose(v, ad, breaks, 2, stream=s)),
        "route_mlp": lambda s: mb.molora_route_mlp(x, W1, b1, W2, b2, 2, stream=s),
        "bucket": lambda s: mb.molora_bucket(r, C, stream=s),
        "gate_dispatch": lambda s: mb.molora_gate_dispatch(v, breaks, ad, 2, stream=s),
        "gate_dispatch_shrink": lambda s: mb.molora_gate_dispatch_shrink(v, breaks, x, A, ad, 2, stream=s)[:3],
        "bucket_shrink": lambda s: mb.molora_bucket_shrink(r, x, A, stream=s),
        "bucket_shrink_small": lambda s: mb.molora_bucket_shrink_small(rs, xs, As, stream=s),
        "shrink_base_small": lambda s: mb.molora_shrink_base_small(rs, xs, W, As, stream=s),
        "shrink": one(lambda s: mb.molora_shrink(x, A, offsets, perm, stream=s)),
        "base_expand": one(lambda s: mb.molora_base_expand(x, W, B, t, offsets, perm, stream=s)),
        "base_expand_dense": one(lambda s: mb.molora_base_expand_dense(x, W, B, td, offsets, perm, stream=s)),
        "apply": one(lambda s: mb.molora_apply(x, W, A, B, r, stream=s)),
        "apply_bucketed": one(lambda s: mb.molora_apply_bucketed(x, W, A, B, offsets, perm, stream=s)),
        "apply_mix": one(lambda s: mb.molora_apply_mix(x, W, A, B, idx, stream=s)),
        "pack_w": one(lambda s: mb.molora_pack_w(W, stream=s)),
        "pack_b": one(lambda s: mb.molora_pack_b(Bs, stream=s)),
    }


@pytest.fixture(scope="module")
def calls():
    return _calls()


NAMES = ["route", "route_vocab", "route_compose", "route_mlp", "bucket", "gate_dispatch", "gate_dispatch_shrink", "bucket_shrink",
         "bucket_shrink_small", "shrink_base_small", "shrink", "base_expand", "base_expand_dense", "apply", "apply_bucketed", "apply_mix",
         "pack_w", "pack_b"]


@pytest.mark.parametrize("name", NAMES)
def test_outputs_are_not_memory_that_the_current_stream_still_uses(calls, name):
    """The current stream is busy, will then write to tensors of the outputs' sizes, and the host has given these
    back already: the call on a side stream must not be handed their memory."""
    import torch
    call = calls[name]
    want = [t.clone() for t in call(None)]
    big = torch.randn(4096, 4096, device="cuda")
    side, out = torch.cuda.Stream(), torch.empty_like(big)
    call(side)
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
    got = call(side)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["route_mlp", "apply", "apply_bucketed", "apply_mix"])
def test_workspaces_of_a_recorded_call_belong_to_the_graph(calls, name):
    import torch
    from paper_2603_15965_amd import binding as mb
    call = calls[name]
    want = [t.clone() for t in call(None)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    call(side)   # the side stream has the memory, given back
    side.synchronize()
    print(f"{name} recorded", flush=True)
    g = mb.Graph(side)
    with g.capture():
        got = call(side)
    sizes = (1 << 12, 1 << 14, 1 << 16, 1 << 18, 1 << 20)
    with torch.cuda.stream(side):   # all that is free on either stream
        fresh = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    side.synchronize()
    fresh += [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    for replay in range(3):
        for t in got:
            t.fill_(99)
        torch.cuda.synchronize()
        g.launch()
        side.synchronize()
        assert all(bool((t == 7).all()) for t in fresh), f"replay {replay} wrote to memory that is another tensor's"
        for a, b in zip(got, want):
            assert torch.equal(a, b), f"replay {replay}"
    g.destroy()
