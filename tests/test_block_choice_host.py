"""The choice of the feed-forward block's kernels, which is made on the host from the sizes (no GPU): the sizes of the GPU
tests reach the kernels that they name, and every kernel that is built is some size's."""
import ctypes
import math
import random

import pytest

import test_gpu_block_kernels as cases
from paper_2603_15965_amd import binding as mb

SIX = {(256, 256, 4), (256, 128, 3), (128, 128, 3), (128, 128, 4), (64, 128, 4), (64, 64, 4)}
SEVEN = {(64, 128, 3), (128, 128, 4), (128, 128, 2), (128, 256, 3), (192, 256, 2), (256, 256, 2), (320, 256, 2)}


def test_the_gpu_tests_reach_what_they_name():
    for tile, sizes in cases.PRODUCTS:
        assert mb.molora_mx_matmul_tile(*sizes) == tile, sizes
    assert {t for t, _ in cases.PRODUCTS if t[2]} == SIX
    for tile, whole, sizes in cases.GATED:
        got = mb.molora_apply_gated_tile(*sizes)
        assert (got[3] == 1) == bool(whole) and (got[2] == 0 if tile is None else got[:3] == tile), sizes
    for which, rows in ((0, cases.DX), (1, cases.DW)):
        for tile, whole, sizes in rows:
            got = mb.molora_gated_backward_tile(*sizes)[which]
            assert got[:3] == tile and (got[3] == 1) == bool(whole), sizes
    for rows in (cases.GATED, cases.DX, cases.DW):   # all tiles in one launch; in slices of K those of up to 192 rows
        assert {t for t, whole, _ in rows if whole and t} == SEVEN
        assert {t for t, whole, _ in rows if not whole} == {t for t in SEVEN if t[0] <= 192}


def test_random_sizes_take_what_is_built():
    rng = random.Random(3)
    lin = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    width = lambda: max(64, lin(64, 12288) // 8 * 8)
    whole, sliced, products = set(), set(), set()
    for _ in range(30000):
        N, d, F = lin(65, 16384), width(), width()
        C, rank = rng.choice([0, lin(1, 256)]), rng.choice([8, 16, 24, 40, 64, 128])
        rank = rank if C else 0
        tiles = [mb.molora_apply_gated_tile(N, d, F, C, rank), *mb.molora_gated_backward_tile(N, d, F, C, rank)]
        for t in tiles:
            (whole if t[3] == 1 else sliced).add(t[:3])
            assert 1 <= t[3] <= 8
        products.add(mb.molora_mx_matmul_tile(N, d, F))
    assert {t for t in whole if t[2]} == SEVEN and sliced == {t for t in SEVEN if t[0] <= 192}
    assert {t for t in whole if not t[2]} == {(64, 32, 0), (64, 64, 0)} and products == SIX


@pytest.mark.parametrize("N,cols", [(1, 16), (64, 16)])
def test_at_most_64_tokens(N, cols):
    rows = (N + 15) // 16 * 16
    for d_out, c in ((8, 16), (4096, 16), (4104, 32), (8192, 32), (8200, 48)):
        assert mb.molora_mx_matmul_tile(N, 512, d_out) == (rows, c, 0)
    for F, c in ((8, 16), (4096, 16), (4104, 32), (8192, 32), (8200, 64)):
        assert mb.molora_apply_gated_tile(N, 512, F, 3, 8)[:3] == (rows, 2 * c, 0)
    assert mb.molora_apply_gated_tile(7, 8192, 9216)[3] > 1   # columns of one round of workgroups and a part


def test_refusals():
    lib = mb.load()
    t = (ctypes.c_int32 * 4)()
    assert lib.molora_mx_matmul_tile(64, 64, 64, None) == -1 and lib.molora_apply_gated_tile(64, 64, 64, 0, 0, None) == -1
    assert lib.molora_gated_backward_tile(64, 64, 64, 0, 0, t, None) == -1 and lib.molora_gated_backward_tile(64, 64, 64, 0, 0, None, t) == -1
    for bad in ((0, 64, 64), (1 << 31, 64, 64), (64, 60, 64), (64, 64, 12)):
        assert lib.molora_mx_matmul_tile(*bad, t) == -1
    for bad in ((0, 64, 64, 0, 0), (64, 60, 64, 0, 0), (64, 64, 12, 0, 0), (64, 64, 64, 0, 8), (64, 64, 64, 2, 12), (1 << 28, 64, 64, 0, 0)):
        assert lib.molora_apply_gated_tile(*bad, t) == -1 and lib.molora_gated_backward_tile(*bad, t, t) == -1
    with pytest.raises(RuntimeError):
        mb.molora_mx_matmul_tile(0, 64, 64)
