"""The sums of the 8-bit floating-point products as the header states them: exact products
summed in fp32 where the result is fp32; where it is bf16, 8 neighbours at a time cut 13 bits
below the largest, an error that the largest products set, not the result.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import plain64 as p64
import plain_experts as pe
from test_gpu_expert_products import dev, same_where_defined, status

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

F32, BF16 = torch.float32, torch.bfloat16


def product(xq, xs, wq, ws, f32):
    M, K = xq.shape
    N = wq.shape[0]
    y, st = torch.empty(M, N, dtype=F32 if f32 else BF16, device="cuda"), status()
    uep.ultraep_expert_matmul_fp8(dev(xq), dev(xs), M, dev(wq), dev(ws), 1, N, K, dev(np.array([0, M])), None, 1,
                                  uep.ULTRAEP_NO_ACT, y, st)
    assert int(st.item()) == 0
    return y.double().cpu().numpy()


def rows_with(values, rows, K):
    """Rows that are zero but for {element: value}, under scales of 1."""
    x = np.zeros((rows, K))
    for k, v in values.items():
        x[:, k] = v
    s = np.zeros((rows, uep.scale_pitch(K)), np.uint8)
    s[:, :-(-K // 128)] = 127
    return pe.e4m3_bits(x), s


@pytest.mark.parametrize("M", [3, 300])
@pytest.mark.parametrize("small", [2, 7, 8, 16, 70, 130])
@pytest.mark.parametrize("f32", [True, False])
def test_a_small_product_beside_large_ones_that_cancel(M, small, f32):
    """448 - 448 + 2^-9: all of it from fp32 sums, and from bf16's where the small product lies
    among 8 others; beside the large ones it may be cut, by 2^-13 of 448 and no more."""
    N, K = 272, 144
    side = rows_with({0: 448.0, 1: 448.0, small: 2.0 ** -9}, M, K), rows_with({0: 1.0, 1: -1.0, small: 1.0}, N, K)
    got = product(*side[0], *side[1], f32)
    if f32 or small >= 8:
        assert (got == 2.0 ** -9).all()
    else:
        assert (np.abs(got - 2.0 ** -9) <= 2.0 ** -13 * 448).all()


@pytest.mark.parametrize("M,N,K", [(5, 64, 1040), (300, 528, 1040), (64, 272, 4096)])
@pytest.mark.parametrize("f32", [True, False])
def test_a_channel_a_hundred_times_larger(M, N, K, f32):
    """A large channel in 512, as activations have them: within the bound that the largest
    products of each 8 set."""
    rng = np.random.default_rng(12)
    x, w = rng.standard_normal((M, K)), rng.standard_normal((N, K)) * K ** -0.5
    x[:, ::512] *= 100
    (xq, xs), (wq, ws) = (pe.quant_blocks(t.astype(np.float32), K) for t in (x, w))
    got = product(xq, xs, wq, ws, f32)
    want, err, _, _ = pe.product(pe.dequantised(xq, xs), pe.dequantised(wq, ws)[None], np.array([0, M]), None, "none",
                                 cut=not f32, taken_to_bf16=f32)
    same_where_defined(got, want, pe.rounded(want, err, f32))
