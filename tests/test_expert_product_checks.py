"""The experts' products with their gradients and in 8-bit floating point, without
a GPU: the plain 64-bit implementations against differences and against torch's
types, the workspace's size, and what the C ABI and the binding refuse before
anything is launched."""
import ctypes
import re

import numpy as np
import pytest
import torch

import paper_2606_04101_amd as uep
import plain_experts as pe
from test_abi import HEADER

E_ = uep.ULTRAEP_EINVAL
BF16, F32, I64, U8 = torch.bfloat16, torch.float32, torch.int64, torch.uint8
NAMES = ["ultraep_expert_matmul_bf16", "ultraep_expert_weight_grad", "ultraep_expert_weight_grad_ws_bytes",
         "ultraep_quant_blocks", "ultraep_expert_matmul_fp8"]


def test_header_and_library_have_the_entry_points():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    lib = ctypes.CDLL(uep.LIB_PATH)
    for n in NAMES:
        assert re.search(rf"\b{n}\s*\(", src) and hasattr(lib, n) and callable(getattr(uep, n))


def test_swiglu_gradient_against_differences():
    """Central differences in 64 bits: h^2 / 6 of the third derivative (below 10 here)
    and rounding 1e-15 / h."""
    rng = np.random.default_rng(5)
    pre, v, h = rng.standard_normal((4, 12)) * 3, rng.standard_normal((4, 6)), 1e-5
    got = pe.swiglu_grad(v, pre)
    for i in range(12):
        hi, lo = pre.copy(), pre.copy()
        hi[:, i] += h
        lo[:, i] -= h
        d = ((pe.swiglu(hi) - pe.swiglu(lo)) * v).sum(axis=1) / (2 * h)
        assert np.abs(d - got[:, i]).max() < 1e-8


def test_product_gradients_against_differences():
    """The transposed product and the weights' gradient are the gradients of sum dy * y,
    which is linear in either: differences are off by rounding alone."""
    rng = np.random.default_rng(6)
    off, of = np.array([0, 3, 3, 7]), [1, 0, 1]
    x, w, dy = rng.standard_normal((7, 5)), rng.standard_normal((2, 4, 5)), rng.standard_normal((7, 4))

    def f(x, w):
        return float((pe.product(x, w, off, of, "none")[0] * dy).sum())
    dx = pe.product(dy, w, off, of, "none", trans=True)[0]
    dw, _ = pe.weight_grad(dy, x, off, of, 2)
    for arr, grad in ((x, dx), (w, dw)):
        for i in np.ndindex(arr.shape):
            old = arr[i]
            arr[i] = old + 1.0
            up = f(x, w)
            arr[i] = old
            assert abs(up - f(x, w) - grad[i]) < 1e-12


def test_e4m3_against_torch():
    bits = torch.arange(256, dtype=torch.int32).to(U8)
    ours, theirs = pe.e4m3_values(), bits.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ours, theirs, equal_nan=True)
    rng = np.random.default_rng(7)
    v = np.concatenate([rng.uniform(-448, 448, 4000), rng.standard_normal(4000) * 0.01, theirs[:127],
                        (theirs[:126] + theirs[1:127]) / 2, [0.0, -0.0, 448, -448, 2.0 ** -10, 2.0 ** -11]])
    assert np.array_equal(pe.e4m3_bits(v), torch.from_numpy(v).to(torch.float8_e4m3fn).view(U8).numpy())


def test_quantised_values_are_within_half_a_step():
    """Within 2^-4 of the value, or of the scaled 2^-6 below which the steps are even."""
    rng = np.random.default_rng(8)
    x = (rng.standard_normal((9, 392)) * np.exp(rng.standard_normal((9, 1)) * 9)).astype(np.float32)
    q, s = pe.quant_blocks(x, 400)
    assert (q[:, 392:] == 0).all() and (s[:, 3] >= 0).all() and s.shape == (9, 4)
    back = pe.dequantised(q[:, :392], s)
    scale = np.repeat(2.0 ** (s.astype(np.float64) - 127), 128, axis=1)[:, :392]
    assert (np.abs(back - x) <= 2.0 ** -4 * np.maximum(np.abs(x), 2.0 ** -6 * scale)).all()
    top = np.abs(np.pad(x, ((0, 0), (0, 120))).reshape(9, 4, 128)).max(axis=2)
    assert (top > 448 * 2.0 ** (s - 128.0)).all()  # half the scale would not do


def test_scale_pitch():
    assert [uep.scale_pitch(k) for k in (8, 128, 512, 513, 7168)] == [4, 4, 4, 8, 56]


def test_weight_grad_workspace_bytes():
    f = uep.ultraep_expert_weight_grad_ws_bytes
    assert f(0, 64, 64, 1) >= 16 and f(1 << 20, 4096, 7168, 5) >= 16
    last = 0
    for M in (0, 1, 100, 4096, 65536, 1 << 20, (1 << 31) - 1):  # one workspace for all batches
        assert f(M, 256, 512, 2) >= last
        last = f(M, 256, 512, 2)
    for bad in [(-1, 64, 64, 1), (1 << 31, 64, 64, 1), (8, 0, 64, 1), (8, 12, 64, 1), (8, 64, 4, 1), (8, 64, 64, 0),
                (8, (1 << 20) + 8, 64, 1), (8, 1 << 20, 1 << 20, 64), (8, 64, 64, (1 << 20) + 1)]:
        assert f(*bad) == 0, bad


def test_bad_arguments_are_refused():
    L, p, odd = uep.lib(), ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 8)  # never dereferenced

    def mm(x=p, M=4, w=p, n_w=2, stride=512, N=16, K=32, trans=0, off=p, of=None, n=2, act=0, pre=None, y=p, type=1,
           st=p):
        return L.ultraep_expert_matmul_bf16(x, M, w, n_w, stride, N, K, trans, off, of, n, act, pre, y, type, st, None)
    for kw in [dict(M=-1), dict(M=1 << 31), dict(M=1 << 30, N=256, stride=8192), dict(n_w=0), dict(N=0), dict(N=12),
               dict(N=(1 << 20) + 8, stride=1 << 30), dict(N=24, stride=768, act=1), dict(K=0), dict(K=20),
               dict(K=(1 << 20) + 8, stride=1 << 30), dict(stride=511), dict(stride=516), dict(stride=504),
               dict(stride=(1 << 40) + 8), dict(trans=2), dict(trans=-1), dict(act=3), dict(act=-1), dict(n=0),
               dict(n=2049), dict(type=2), dict(x=None), dict(x=odd), dict(w=None), dict(w=odd), dict(off=None),
               dict(pre=p), dict(act=1, pre=odd), dict(act=2), dict(act=2, pre=odd), dict(y=None), dict(y=odd),
               dict(st=None)]:
        assert mm(**kw) == E_, kw
    assert mm(M=0, x=None, y=None) == uep.ULTRAEP_OK

    def wg(dy=p, x=p, M=4, N=16, K=32, off=p, of=None, n=2, n_w=2, stride=512, acc=0, dw=p, type=0, ws=None, nb=0, st=p):
        return L.ultraep_expert_weight_grad(dy, x, M, N, K, off, of, n, n_w, stride, acc, dw, type, ws, nb, st, None)
    for kw in [dict(M=-1), dict(M=1 << 31), dict(N=0), dict(N=20), dict(K=0), dict(K=36), dict(n=0), dict(n=2049),
               dict(n_w=0), dict(n_w=(1 << 20) + 1), dict(N=1 << 20, K=1 << 20, stride=1 << 40, n_w=16),
               dict(stride=508), dict(stride=516), dict(acc=2), dict(acc=-1), dict(type=2), dict(dy=None), dict(dy=odd),
               dict(x=None), dict(x=odd), dict(dw=None), dict(dw=odd), dict(off=None), dict(st=None), dict(ws=p, nb=0),
               dict(ws=odd, nb=1 << 30)]:
        assert wg(**kw) == E_, kw

    def quant(x=p, type=1, rows=4, K=16, ld=16, q=p, ldq=16, scale=p):
        return L.ultraep_quant_blocks(x, type, rows, K, ld, q, ldq, scale, None)
    for kw in [dict(type=2), dict(rows=-1), dict(rows=1 << 31), dict(K=0), dict(K=12), dict(ld=8), dict(ld=20),
               dict(ld=(1 << 20) + 8), dict(ldq=8), dict(ldq=24), dict(ldq=(1 << 20) + 16), dict(x=None), dict(x=odd),
               dict(q=None), dict(q=odd), dict(scale=None), dict(scale=ctypes.c_void_p(4098))]:
        assert quant(**kw) == E_, kw
    assert quant(rows=0) == uep.ULTRAEP_OK

    def m8(xq=p, xs=p, M=4, wq=p, ws=p, n_w=2, N=16, K=32, off=p, of=None, n=2, act=0, y=p, type=1, st=p):
        return L.ultraep_expert_matmul_fp8(xq, xs, M, wq, ws, n_w, N, K, off, of, n, act, y, type, st, None)
    two = ctypes.c_void_p(4098)
    for kw in [dict(M=-1), dict(M=1 << 31), dict(M=1 << 30, N=256), dict(n_w=0), dict(N=0), dict(N=12), dict(N=8, act=1),
               dict(N=(1 << 20) + 8), dict(act=2), dict(act=-1), dict(K=0), dict(K=24), dict(K=(1 << 20) + 16), dict(n=0),
               dict(n=2049), dict(type=3), dict(xq=None), dict(xq=odd), dict(xs=None), dict(xs=two), dict(wq=None),
               dict(wq=odd), dict(ws=None), dict(ws=two), dict(off=None), dict(y=None), dict(y=odd), dict(st=None)]:
        assert m8(**kw) == E_, kw
    assert m8(M=0) == uep.ULTRAEP_OK


def test_outputs_in_the_place_of_inputs_are_refused():
    L = uep.lib()
    a, b, c, d, off, st = (ctypes.c_void_p(4096 * i) for i in range(1, 7))  # never dereferenced

    def mm(x, w, pre, y, act, type_):
        return L.ultraep_expert_matmul_bf16(x, 4, w, 1, 512, 16, 32, 0, off, None, 1, act, pre, y, type_, st, None)
    none, glu, grad = uep.ULTRAEP_NO_ACT, uep.ULTRAEP_SWIGLU, uep.ULTRAEP_SWIGLU_GRAD
    for args in [(a, b, None, a, none, 1), (a, b, None, b, none, 1), (a, b, c, c, glu, 1), (a, b, a, c, glu, 1),
                 (a, b, b, c, glu, 1), (a, b, c, c, grad, 0), (a, b, c, a, grad, 1)]:
        assert mm(*args) == E_, args

    def wg(dy, x, dw, ws):
        return L.ultraep_expert_weight_grad(dy, x, 4, 16, 32, off, None, 1, 1, 512, 0, dw, 0, ws, 1 << 20, st, None)
    for args in [(a, b, a, None), (a, b, b, None), (a, b, c, a), (a, b, c, b), (a, b, c, c)]:
        assert wg(*args) == E_, args
    for x, q, s in [(a, a, b), (a, b, a), (a, b, b)]:
        assert L.ultraep_quant_blocks(x, 1, 4, 16, 16, q, 16, s, None) == E_
    for y in (a, b, c, d):
        assert L.ultraep_expert_matmul_fp8(a, b, 4, c, d, 1, 16, 32, off, None, 1, 0, y, 1, st, None) == E_


def t(n, dtype=torch.int32):
    return torch.zeros(n, dtype=dtype)


def test_binding_refuses_small_or_wrong_tensors():
    M, N, K, n_w, stride = 4, 16, 32, 2, 520
    off = t(3, I64)
    a = dict(x=t(M * K, BF16), M=M, w=t(stride + N * K, BF16), n_w=n_w, w_stride=stride, N=N, K=K, trans=False,
             block_off=off, block_w=None, n_block=2, act=uep.ULTRAEP_SWIGLU, pre=t(M * N, BF16), y=t(M * N // 2, BF16),
             status=t(1))
    grad = dict(a, act=uep.ULTRAEP_SWIGLU_GRAD, pre=t(M * 2 * N, BF16), y=t(M * 2 * N, F32), trans=True)
    for base, name, bad in [
            (a, "x", t(M * K - 1, BF16)), (a, "x", t(M * K, F32)), (a, "w", t(stride + N * K - 1, BF16)),
            (a, "block_off", t(2, I64)), (a, "block_off", t(3)), (a, "block_w", t(1)), (a, "pre", t(M * N - 1, BF16)),
            (a, "pre", t(M * N, F32)), (a, "y", t(M * N // 2 - 1, BF16)), (a, "y", t(M * N, torch.float16)),
            (a, "status", None), (grad, "pre", t(M * 2 * N - 1, BF16)), (grad, "pre", None),
            (grad, "y", t(M * 2 * N - 1, F32))]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_expert_matmul_bf16(*{**base, name: bad}.values())
    g = dict(dy=t(M * N, BF16), x=t(M * K, BF16), M=M, N=N, K=K, block_off=off, block_w=None, n_block=2, n_w=n_w,
             dw_stride=stride, accumulate=True, dw=t(stride + N * K, F32), ws=None, status=t(1))
    for name, bad in [("dy", t(M * N - 1, BF16)), ("x", t(M * K, F32)), ("block_off", t(1, I64)), ("block_w", t(1)),
                      ("dw", t(stride + N * K - 1, F32)), ("dw", t(stride + N * K, torch.float16)), ("status", None)]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_expert_weight_grad(*{**g, name: bad}.values())
    q = dict(x=t(3 * 32 + 24, BF16), rows=4, K=24, ld=32, q=t(4 * 32, U8), ldq=32, scale=t(16, U8))
    for name, bad in [("x", t(3 * 32 + 23, BF16)), ("x", t(4 * 32, torch.float16)), ("q", t(4 * 32 - 1, U8)),
                      ("q", t(4 * 32)), ("scale", t(15, U8)), ("scale", t(16, F32))]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_quant_blocks(*{**q, name: bad}.values())
    m = dict(xq=t(4 * 528, U8), x_scale=t(4 * 8, U8), M=4, wq=t(2 * 16 * 528, U8), w_scale=t(2 * 16 * 8, U8), n_w=2, N=16,
             K=528, block_off=off, block_w=None, n_block=2, act=1, y=t(4 * 8, BF16), status=t(1))
    for name, bad in [("xq", t(4 * 528 - 1, U8)), ("x_scale", t(31, U8)), ("wq", t(2 * 16 * 528 - 1, U8)),
                      ("w_scale", t(255, U8)), ("w_scale", t(256, F32)), ("block_off", t(3)), ("block_w", t(1)),
                      ("y", t(31, BF16)), ("status", t(0))]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_expert_matmul_fp8(*{**m, name: bad}.values())


def test_native_half_declines_host_tensors():
    n = uep._load_native()
    assert n.quant_blocks(t(16, F32), 1, 16, 16, t(16, U8), 16, t(4, U8), 0) is None
    assert n.expert_matmul_bf16(t(8, BF16), 1, t(64, BF16), 1, 64, 8, 8, 0, t(2, I64), None, 1, 0, None, t(8, BF16), t(1),
                                0) is None
    assert n.expert_weight_grad(t(8, BF16), t(8, BF16), 1, 8, 8, t(2, I64), None, 1, 1, 64, 0, t(64, F32), None, t(1),
                                0) is None
