"""The 256 x 256 tiles of the experts' products and of their weights' gradient, which carry the
large calls: many steps of the common index with a remainder (so that the buffers go round, and
in 8 bits the words of scales), several tiles a workgroup and a last round by quarters, of
every type and act.  Against torch in 64 bits, within the bounds that plain_experts derives.
That a case takes these tiles is asked of the library's own rule.  Needs an MI355X."""
import ctypes

import numpy as np
import pytest
import torch

import plain64 as p64
import plain_experts as pe

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep
    ACTS = {"none": uep.ULTRAEP_NO_ACT, "swiglu": uep.ULTRAEP_SWIGLU, "swiglu_grad": uep.ULTRAEP_SWIGLU_GRAD}

F32, F64, BF16, U8, I32 = torch.float32, torch.float64, torch.bfloat16, torch.uint8, torch.int32
U = {F32: p64.U32, BF16: p64.U16}
START, TAIL = 3, 5  # rows before the blocks and behind them


def rows_of(sizes):
    off = START + np.concatenate([[0], np.cumsum(sizes)])
    return off.tolist(), int(off[-1]) + TAIL


def quarters(sizes, n_col):
    """Tiles of the last round, where quarters take it."""
    last = sum(-(-s // 256) for s in sizes) * n_col % 256
    return last if 0 < last <= 64 else 0


def takes_large(M, n, N, K, eight, trans, act, dtype):
    return uep.lib().uep_product_tile(ctypes.c_int64(M), n, N, K, int(eight), int(trans), ACTS[act],
                                      uep.ULTRAEP_F32 if dtype == F32 else uep.ULTRAEP_BF16) == 0


def randn(g, *shape, spoil=None):
    t = torch.randn(*shape, device="cuda", generator=g).to(BF16)
    if spoil:
        t[:START] = t[-TAIL:] = float("nan")
    return t


def activate(v, dv, act, pre=None):
    """pe.activate on the GPU."""
    if act == "none":
        return v, dv
    if act == "swiglu":
        (a, b), (da, db) = v.chunk(2, 1), dv.chunk(2, 1)
        s = a * torch.sigmoid(a)
        y = s * b
        return y, 1.1 * da * (b.abs() + db) + s.abs() * db + (16 + 3 * a.abs()) * p64.U32 * y.abs() + pe.TINY * (1 + b.abs())
    a, b = pre.chunk(2, 1)
    s = torch.sigmoid(a)
    y = torch.cat([v * b * s * (1 + a * (1 - s)), v * a * s], 1)
    size = torch.cat([b.abs() * s * (1 + a.abs() * (1 - s)), a.abs() * s], 1)
    a2, v2, dv2 = (torch.cat([t, t], 1) for t in (a, v, dv))
    return y, size * (dv2 + (20 + 3 * a2.abs()) * p64.U32 * v2.abs()) + pe.TINY * (1 + v2.abs())


def near(got, want, err, dtype):
    """Within the bound and the rounding of the result, half a step of its type."""
    ok = (got.double() - want).abs() <= err + U[dtype] * (want.abs() + err) + 1e-37
    assert ok.all(), (int((~ok).sum()), torch.nonzero(~ok)[:5].tolist())


def eights(x):
    x = torch.nn.functional.pad(x.abs(), (0, -x.shape[1] % 8))
    return x.view(x.shape[0], -1, 8).amax(2)


def check(sizes, off, x, w, act, dtype, y, pre, cut=False):
    """Block by block; w(g): weights [N][K] of block g in 64 bits."""
    kept = pre is not None and act == "swiglu"
    K = x(0, 1).shape[1]
    assert not torch.isnan(y[START:-TAIL]).any()
    for t in (y, pre) if kept else (y,):
        assert (t[:START] == 3).all() and (t[-TAIL:] == 3).all()
    for g in range(len(sizes)):
        lo, hi = off[g], off[g + 1]
        if hi == lo:
            continue
        xs, ws = x(lo, hi), w(g)
        v = xs @ ws.t().contiguous()
        dv = 2 * K * p64.U32 * (xs.abs() @ ws.abs().t().contiguous()) + 1e-37
        if cut:
            dv += 7 * 2.0 ** -13 * (eights(xs) @ eights(ws).t().contiguous())
        near(y[lo:hi], *activate(v, dv, act, pre[lo:hi].double() if act == "swiglu_grad" else None), dtype)
        if kept:
            near(pre[lo:hi], v, dv, BF16)


CASES = [([2000, 2230], 4088), ([4100, 3900, 0, 280], 4096)]  # a round and quarters; two rounds and quarters


@pytest.mark.parametrize("K", [344, 520])
@pytest.mark.parametrize("sizes,N", CASES)
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("act", ["none", "swiglu", "swiglu_grad"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_bf16_products(sizes, N, K, trans, act, dtype):
    N = N // 16 * 16 if act == "swiglu" else N
    (off, M), n = rows_of(sizes), len(sizes)
    assert takes_large(M, n, N, K, False, trans, act, dtype)
    assert quarters(sizes, -(-N // 256))
    g = torch.Generator(device="cuda").manual_seed(K)
    x, w = randn(g, M, K, spoil=True), randn(g, n, *((K, N) if trans else (N, K)))
    width = {"none": N, "swiglu": N // 2, "swiglu_grad": 2 * N}[act]
    y = torch.full((M, width), 3.0, dtype=dtype, device="cuda")
    pre = {"none": None, "swiglu": torch.full((M, N), 3.0, dtype=BF16, device="cuda"),
           "swiglu_grad": randn(g, M, 2 * N) if act == "swiglu_grad" else None}[act]
    of = [(i + 1) % n for i in range(n)]
    args = (x, M, w, n, N * K, N, K, trans, torch.tensor(off, device="cuda"), torch.tensor(of, dtype=I32, device="cuda"), n,
            ACTS[act])
    st = torch.zeros(1, dtype=I32, device="cuda")
    uep.ultraep_expert_matmul_bf16(*args, pre, y, st)
    assert int(st.item()) == 0
    check(sizes, off, lambda lo, hi: x[lo:hi].double(), lambda b: (w[of[b]].t().contiguous() if trans else w[of[b]]).double(),
          act, dtype, y, pre)
    first = y.clone()
    for _ in range(2):  # again, with the same bits
        uep.ultraep_expert_matmul_bf16(*args, pre, y, st)
        assert torch.equal(y, first)
    if act == "swiglu_grad" and dtype == BF16:  # in the place of what it reads
        pre[:START] = pre[-TAIL:] = 3.0
        uep.ultraep_expert_matmul_bf16(*args, pre, pre, st)
        assert torch.equal(pre, first)


def quantised(x):
    rows, K = x.shape
    q = torch.empty(rows, K, dtype=torch.float8_e4m3fn, device="cuda")
    s = torch.empty(rows, uep.scale_pitch(K), dtype=U8, device="cuda")
    uep.ultraep_quant_blocks(x, rows, K, K, q, K, s)
    power = torch.arange(K, device="cuda") // 128
    return q, s, torch.ldexp(q.to(F32).double(), s[:, power].to(I32) - 127)


@pytest.mark.parametrize("K", [528, 1040, 1424])  # 5, 9 and 12 steps: 2 and 3 words of scales
@pytest.mark.parametrize("sizes,N", CASES)
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_fp8_products(sizes, N, K, act):
    N = N // 16 * 16
    (off, M), n = rows_of(sizes), len(sizes)
    assert takes_large(M, n, N, K, True, False, act, BF16) and quarters(sizes, -(-N // 256))
    g = torch.Generator(device="cuda").manual_seed(K)
    # scales that differ from block to block
    spread = torch.exp2(torch.randint(-6, 7, (1, -(-K // 128)), device="cuda", generator=g).float()).repeat_interleave(128, 1)
    x = torch.randn(M, K, device="cuda", generator=g) * spread[:, :K]
    w = torch.randn(n * N, K, device="cuda", generator=g) / spread[:, :K]
    xq, xs, x64 = quantised(x)
    wq, ws, w64 = quantised(w)
    y = torch.full((M, N // 2 if act == "swiglu" else N), 3.0, dtype=BF16, device="cuda")
    st = torch.zeros(1, dtype=I32, device="cuda")
    args = (xq, xs, M, wq, ws, n, N, K, torch.tensor(off, device="cuda"), None, n, ACTS[act], y, st)
    uep.ultraep_expert_matmul_fp8(*args)
    assert int(st.item()) == 0
    w64 = w64.view(n, N, K)
    check(sizes, off, lambda lo, hi: x64[lo:hi], lambda b: w64[b], act, BF16, y, None, cut=True)
    first = y.clone()
    for _ in range(2):
        uep.ultraep_expert_matmul_fp8(*args)
        assert torch.equal(y, first)


@pytest.mark.parametrize("K", [528, 1040, 1424])
def test_fp8_products_of_small_integers_are_exact(K):
    """Under scales of 1/4 to 4 that cancel between the sides: every element that another
    place, or a scale that another step brings, is seen."""
    sizes, N = CASES[0]
    (off, M), n = rows_of(sizes), len(sizes)
    assert takes_large(M, n, N, K, True, False, "none", BF16)
    g = torch.Generator(device="cuda").manual_seed(K)
    pitch = uep.scale_pitch(K)
    x, w = (torch.randint(-3, 4, (r, K), device="cuda", generator=g).float() for r in (M, n * N))
    power = torch.randint(-2, 3, (pitch,), device="cuda", generator=g)
    xs, ws = (p.to(U8).repeat(r, 1).contiguous() for p, r in ((127 + power, M), (127 - power, n * N)))
    y = torch.empty(M, N, dtype=BF16, device="cuda")
    st = torch.zeros(1, dtype=I32, device="cuda")
    uep.ultraep_expert_matmul_fp8(x.to(torch.float8_e4m3fn), xs, M, w.to(torch.float8_e4m3fn), ws, n, N, K,
                                  torch.tensor(off, device="cuda"), None, n, 0, y, st)
    for b in range(n):
        want = x[off[b]:off[b + 1]].double() @ w[b * N:(b + 1) * N].double().t().contiguous()
        assert torch.equal(y[off[b]:off[b + 1]], want.to(BF16))


GRADS = [  # sizes, block's weights, weights, N, K: whole and ragged tiles, one round and two, parts
    ([1100, 0, 500], [1, 0, 0], 2, 4088, 2040), ([300, 150], [0, 1], 2, 4096, 2048),
    ([900, 1, 1301, 1500], [2, 0, 3, 1], 4, 4088, 2040), ([65, 700, 64, 1000, 0, 500, 1500], [0, 0, 1, 3, 2, 1, 3], 4, 4096, 2048)]


def check_weight_grad(sizes, of, n_w, N, K, dtype, accumulate, parts):
    (off, M), n, gap = rows_of(sizes), len(sizes), 16
    assert uep.lib().uep_weight_grad_large(ctypes.c_int64(M), N, K, n_w, uep.ULTRAEP_F32 if dtype == F32 else uep.ULTRAEP_BF16,
                                           int(parts))
    ws = None
    if parts:
        ws = torch.full((uep.ultraep_expert_weight_grad_ws_bytes(M, N, K, n_w),), 255, dtype=U8, device="cuda")
        assert ws.numel() > 16
    g = torch.Generator(device="cuda").manual_seed(N + K)
    dy, x = randn(g, M, N, spoil=True), randn(g, M, K, spoil=True)
    old = torch.full((n_w, N * K + gap), 7.0, dtype=dtype, device="cuda")
    if accumulate:
        old[:, :N * K] = 3 * torch.randn(n_w, N * K, device="cuda", generator=g)
    args = (dy, x, M, N, K, torch.tensor(off, device="cuda"), torch.tensor(of, dtype=I32, device="cuda"), n, n_w, N * K + gap,
            accumulate)
    st, results = torch.zeros(1, dtype=I32, device="cuda"), []
    for _ in range(3):
        dw = old.clone()
        uep.ultraep_expert_weight_grad(*args, dw, ws, st)
        results.append(dw)
    assert int(st.item()) == 0 and torch.equal(results[0], results[1]) and torch.equal(results[0], results[2])
    assert (dw[:, N * K:] == 7).all()
    for u in range(n_w):
        want = torch.zeros(N, K, dtype=F64, device="cuda")
        mag, rows = torch.zeros_like(want), 0
        for b in range(n):
            lo, hi = off[b], off[b + 1]
            if of[b] == u and hi > lo:
                a, c = dy[lo:hi].double().t().contiguous(), x[lo:hi].double()
                want += a @ c
                mag += a.abs() @ c.abs()
                rows += hi - lo
        err = 2 * (rows + 2) * p64.U32 * mag + 1e-37
        if accumulate:
            want += old[u, :N * K].view(N, K).double()
            err += p64.U32 * (want.abs() + err)
        near(dw[u, :N * K].view(N, K), want, err, dtype)


@pytest.mark.parametrize("case", range(len(GRADS)))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad(case, dtype, accumulate):
    check_weight_grad(*GRADS[case], dtype, accumulate, parts=False)


@pytest.mark.parametrize("sizes,of,n_w,N,K", [([5000, 3192], [0, 0], 1, 2040, 2032), ([9000, 0, 6900, 500], [0, 1, 0, 1], 2, 2040, 1016)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad_in_parts(sizes, of, n_w, N, K, dtype, accumulate):
    check_weight_grad(sizes, of, n_w, N, K, dtype, accumulate, parts=True)
