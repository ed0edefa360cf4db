"""The sizes of the GPU tests of the experts' products, asked of the library's own rules: each
kind of product meets every tile that it can take, so that another rule cannot leave one
untested unseen.  No GPU is needed."""
import ctypes

import pytest

import paper_2606_04101_amd as uep
import test_gpu_expert_large_tiles as large
import test_gpu_expert_products as gpu

NONE, GLU, GRAD = uep.ULTRAEP_NO_ACT, uep.ULTRAEP_SWIGLU, uep.ULTRAEP_SWIGLU_GRAD
F32, BF16 = uep.ULTRAEP_F32, uep.ULTRAEP_BF16
TILES, MANY = gpu.TILES, gpu.MANY
TILES8, MANY8 = ([(s, n // 16 * 16, k // 16 * 16) for s, n, k in c] for c in (TILES, MANY))
LARGE = [(s, n, k) for s, n in large.CASES for k in (344, 520)]
LARGE8 = [(s, n // 16 * 16, 1040) for s, n in large.CASES]


def taken(cases, eight, trans, act, type):
    out = set()
    for sizes, N, K in cases:
        t = uep.lib().uep_product_tile(ctypes.c_int64(sum(sizes)), len(sizes), N, K, eight, trans, act, type)
        out.add((t, K * (1 if eight else 2) >= 4096) if t >= 4 else t)
    return out


THIN = {(t, deep) for t in (4, 5, 6) for deep in (False, True)}


@pytest.mark.parametrize("cases,eight,trans,act,type,want", [
    (gpu.SHAPES + TILES + MANY + LARGE, 0, 0, NONE, BF16, {0, 1, 2, 3} | THIN),
    (gpu.SHAPES + TILES + MANY + LARGE, 0, 0, GLU, BF16, {0, 1, 2, 3} | THIN),
    (gpu.SHAPES + MANY + LARGE, 0, 0, GRAD, BF16, {0, 1, 2, 3}),
    (gpu.SHAPES + TILES + MANY + LARGE, 0, 1, NONE, BF16, {0, 1, 2, 3}),
    (gpu.SHAPES + MANY + LARGE, 0, 1, GLU, BF16, {0, 1, 2, 3}),
    (gpu.SHAPES + TILES + MANY + LARGE, 0, 1, GRAD, BF16, {0, 1, 2, 3}),
    (gpu.SHAPES8 + MANY8 + LARGE8, 1, 0, NONE, BF16, {0, 2, 3} | THIN),
    (gpu.SHAPES8 + MANY8 + LARGE8, 1, 0, GLU, BF16, {0, 2, 3} | THIN),
    (gpu.SHAPES8 + MANY8, 1, 0, NONE, F32, {1, 2, 3} | THIN)])
def test_every_tile_is_met(cases, eight, trans, act, type, want):
    got = taken(cases, eight, trans, act, type)
    assert got >= want, want - got


def test_the_largest_tiles_take_whole_rounds_and_quarters():
    """(The quarters are chosen on the device, by the same count.)"""
    assert all(large.quarters(s, -(-n // 256)) for s, n in large.CASES)
    assert any(sum(-(-r // 256) for r in s) * -(-n // 256) >= 512 for s, n in large.CASES)


def test_both_tiles_of_the_weights_gradient():
    def takes(M, N, K, n_w, parts):
        return [uep.lib().uep_weight_grad_large(ctypes.c_int64(M), N, K, n_w, t, parts) for t in (F32, BF16)]
    for sizes, _, n_w, N, K in large.GRADS:
        assert takes(sum(sizes) + 8, N, K, n_w, 0) == [1, 1]
    assert takes(950, 264, 520, 1, 0) == takes(950, 264, 520, 1, 1) == [0, 0]
