"""The SwiGLU of the experts' products to fp32, as accurate as the header states: by the hardware's
exp2 and reciprocal, (1.25 |v| + 6) 2^-24 of silu(v), whose exponential is off by
(1.23 |v| + 2) 2^-24, the sum by one rounding, the reciprocal by two and the product by one.
Needs an MI355X."""
import numpy as np
import pytest
import torch

import plain64 as p64
import plain_experts as pe
from test_gpu_expert_products import dev, dev16, status

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

F32, BF16 = torch.float32, torch.bfloat16


def gates():
    """Rows whose first element is a gate (of bf16, 2^-20 to 120, of both signs), whose second is 1."""
    g = p64.bf16(np.concatenate([np.geomspace(2.0 ** -20, 120, 4000), np.linspace(0.1, 95, 4000)]).astype(np.float32))
    x = np.zeros((16000, 16), np.float32)
    x[:, 0], x[:, 1] = np.concatenate([g, -g]), 1.0
    return x


def check(y, v):
    y = y.double().cpu().numpy()
    assert (y == y[:, :1]).all()
    y, v = y[:, 0], v.astype(np.float64)
    want = pe.silu(v)
    assert (np.abs(y - want) <= (1.25 * np.abs(v) + 6) * p64.U32 * np.abs(want))[v >= -87.3].all()
    assert (np.abs(y) < 2e-36)[v < -87.3].all()


def weights(N, K):
    w = np.zeros((1, N, K), np.float32)
    w[0, :N // 2, 0] = w[0, N // 2:, 1] = 1.0
    return w


@pytest.mark.parametrize("rows", [16000, 40])
def test_bf16(rows):
    x = gates()[::16000 // rows]
    (M, K), N = x.shape, 32
    y = torch.empty(M, N // 2, device="cuda")
    uep.ultraep_expert_matmul_bf16(dev16(x), M, dev16(weights(N, K)), 1, N * K, N, K, False, dev(np.array([0, M])), None, 1,
                                   uep.ULTRAEP_SWIGLU, None, y, status())
    check(y, x[:, 0])


@pytest.mark.parametrize("rows", [16000, 40])
def test_fp8(rows):
    """The gates as e4m3 hold them."""
    x = gates()[::16000 // rows]
    (M, K), N = x.shape, 32
    xq, xs = pe.quant_blocks(x, K)
    v = pe.dequantised(xq, xs)
    x[:, 0] = v[:, 0]
    keep = v[:, 1] == 1.0  # (beside a large gate e4m3 may not hold the 1)
    wq, ws = pe.quant_blocks(weights(N, K)[0], K)
    y, st = torch.empty(M, N // 2, device="cuda"), status()
    uep.ultraep_expert_matmul_fp8(dev(xq), dev(xs), M, dev(wq), dev(ws), 1, N, K, dev(np.array([0, M])), None, 1,
                                  uep.ULTRAEP_SWIGLU, y, st)
    assert int(st.item()) == 0 and keep.mean() > 0.9
    check(y[torch.from_numpy(keep).cuda()], x[keep, 0])
