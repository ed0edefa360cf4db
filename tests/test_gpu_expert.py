"""The row quantisation, the 8-bit expert products and the combine's backward
pass on the GPU against the plain 64-bit implementations.  Needs an MI355X.

Quantised values, scales and dy are exact (one order of fp32 operations).  A
product's sum is exact in 32-bit integers, so y is off by the roundings that
plain64.expert_matmul counts, and by half an ulp of its own type.  dgate is a sum
of H fp32 products: at most H + 1 roundings of the sum of their magnitudes."""
import numpy as np
import pytest
import torch

import plain64 as p64

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

I32, I64, F32 = torch.int32, torch.int64, torch.float32


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def status():
    return torch.zeros(1, dtype=I32, device="cuda")


# ------------------------------------------------------------------ quant_rows

@pytest.mark.parametrize("rows,K,ld,ldq", [
    (1, 8, 8, 16), (1, 16, 16, 16), (3, 24, 40, 32), (65, 520, 520, 528), (257, 2888, 2896, 2896),
    (40, 7168, 7168, 7168), (9, 12288, 12296, 12304), (5, 16392, 16392, 16400), (3, 65536, 65536, 65536),
    (2, 131080, 131080, 131104), (1000, 64, 72, 128)])
@pytest.mark.parametrize("bf16", [True, False])
def test_quant_rows(rows, K, ld, ldq, bf16):
    rng = np.random.default_rng(rows * K)
    x = (rng.standard_normal((rows, ld)) * np.exp(2 * rng.standard_normal((rows, 1)))).astype(np.float32)
    x[:, K:] = np.nan  # what lies between rows is not looked at
    if rows > 4:
        x[1, :K] = 0
        x[2, :K] *= np.float32(1e-35)   # below the smallest scale
        x[3, :K] *= np.float32(1e30)
    if bf16:
        x = p64.bf16(x)
    q = torch.full((rows * ldq + 64,), 55, dtype=torch.int8, device="cuda")
    s = torch.full((rows + 8,), 5., device="cuda")
    uep.ultraep_quant_rows(dev(p64.bf16_bits(x).view(np.int16) if bf16 else x), rows, K, ld, q, ldq, s)
    rq, rs = p64.quant_rows(x[:, :K])
    got = q[:rows * ldq].cpu().numpy().reshape(rows, ldq)
    assert np.array_equal(got[:, :K], rq) and (got[:, K:] == 0).all()
    assert np.array_equal(s[:rows].cpu().numpy(), rs)
    assert (q[rows * ldq:] == 55).all() and (s[rows:] == 5).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_quant_rows_of_other_numbers(bf16):
    """Infinities, NaN, the type's largest values, zeros of both signs, exact
    halves (to even)."""
    x = np.zeros((8, 32), np.float32)
    x[0, 3] = np.inf
    x[1, 31] = -np.inf
    x[2, 0] = np.nan
    x[3] = -0.0
    x[4] = np.linspace(-1, 1, 32) * 3e38
    x[5, :6] = [127, 0.5, 1.5, 2.5, -0.5, -1.5]
    x[6, 0] = 2.0 ** -100
    x[7, 0] = 2.0 ** -99
    if bf16:
        x = p64.bf16(x)
    q, s = torch.empty(8, 32, dtype=torch.int8, device="cuda"), torch.empty(8, device="cuda")
    uep.ultraep_quant_rows(dev(p64.bf16_bits(x).view(np.int16) if bf16 else x), 8, 32, 32, q, 32, s)
    rq, rs = p64.quant_rows(x)
    assert np.array_equal(q.cpu().numpy(), rq)
    assert np.array_equal(s.cpu().numpy(), rs, equal_nan=True)
    assert q[5, :6].tolist() == [127, 0, 2, 2, 0, -2] and q[7, 0] == 127 and float(s[6]) == 0


def test_quant_rows_offsets_past_32_bits():
    rows, K = 300_001, 8192
    x = torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, K, device="cuda").to(torch.bfloat16)
    q, s = torch.empty(rows, K, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    uep.ultraep_quant_rows(x, rows, K, K, q, K, s)
    rq, rs = p64.quant_rows(x[-3:].float().cpu().numpy())
    assert np.array_equal(q[-3:].cpu().numpy(), rq) and np.array_equal(s[-3:].cpu().numpy(), rs)
    assert not q[:-3].any() and not s[:-3].any()


# --------------------------------------------------------------- expert_matmul

def products(M, N, K, sizes, n_w, act, f32, seed=0, of=None, start=0, extreme=False):
    rng = np.random.default_rng(seed)
    if extreme:
        xq = np.full((M, K), 127, np.int8)
        wq = np.full((n_w, N, K), -127, np.int8)
    else:
        xq = rng.integers(-127, 128, (M, K)).astype(np.int8)
        wq = rng.integers(-127, 128, (n_w, N, K)).astype(np.int8)
    xs = (rng.random(M) * 0.02 + 0.001).astype(np.float32)
    ws = (rng.random((n_w, N)) * 0.02 + 0.001).astype(np.float32) / np.float32(np.sqrt(K))
    off = start + np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    n_out = N // 2 if act else N
    y = torch.full((M, n_out), 3.0, dtype=F32 if f32 else torch.bfloat16, device="cuda")
    st = status()
    uep.ultraep_expert_matmul(dev(xq), dev(xs), M, dev(wq), dev(ws), n_w, N, K, dev(off),
                              None if of is None else dev(np.array(of, np.int32)), len(sizes), act, y, st)
    assert int(st.item()) == 0
    want, rel = p64.expert_matmul(xq, xs, wq, ws, off, of, act)
    got = y.double().cpu().numpy()
    inside = np.zeros(M, bool)
    inside[off[0]:off[-1]] = True
    assert (got[~inside] == 3).all()  # rows outside the blocks are left alone
    tol = (rel + (0 if f32 else 1.01 * p64.U16)) * np.abs(want) + 1e-37
    assert (np.abs(got - want)[inside] <= tol[inside]).all()


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 129, 200, 257, 511, 700])
def test_matmul_rows(M, act, f32):
    products(M, 208, 400, [M], 1, act, f32, seed=M)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("N,K", [(16, 16), (16, 48), (32, 64), (48, 80), (64, 112), (112, 128), (144, 144), (256, 256),
                                 (272, 1040), (528, 272), (1024, 528), (16, 4096), (2064, 32)])
@pytest.mark.parametrize("M", [3, 40, 300])
def test_matmul_shapes(N, K, M, act):
    products(M, N, K, [M], 1, act, False, seed=N + K)


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("sizes,of", [
    ([5, 0, 9, 1], None), ([0, 0, 0, 0], None), ([300, 1, 0, 257, 64], [4, 0, 3, 3, 1]), ([1] * 40, None),
    ([0] * 30 + [70] + [0] * 10, None), ([128, 256, 128, 512], None), ([33, 65, 129, 17], [2, 2, 2, 2]),
    ([3, 0] * 200, list(range(400))), ([700, 2, 2, 2, 2, 2], None)])
def test_matmul_blocks(sizes, of, act):
    n_w = len(sizes) if of is None or len(of) > 8 else 6
    products(max(1, sum(sizes)), 144, 160, sizes, n_w, act, False, seed=len(sizes), of=of)


# (blocks' rows, N, K) that reach each of the tile shapes: few rows with K shared by
# four waves and by two, 64, 128 and 256 rows a tile; with ends inside tiles and steps
WIDE = [([3, 0, 40], 16416, 4112), ([45], 16400, 4112), ([41], 16400, 176), ([20], 16400, 4096), ([13, 9, 20], 5472, 272),
        ([9, 70, 33, 50, 1, 0, 64, 65] * 5, 1040, 144), ([2050], 2064, 80), ([700, 64, 65, 300, 900], 1552, 400),
        ([3500, 130], 4112, 144), ([257, 1000, 2300], 4112, 48), ([1030, 255, 256, 900, 5], 8208, 1040)]


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("sizes,N,K", WIDE)
def test_matmul_tiles(sizes, N, K, act):
    products(sum(sizes), N, K, sizes, len(sizes), act, N % 32 == 0 or K == 144, seed=N)


# several rounds of 256-row tiles over 256 workgroups, the last of them whole (442 and 680
# tiles) or by quarters (289, 306, 279, 320), some of those with no rows or no channels
ROUNDS = [([130, 5000, 3, 900], 4112, 80), ([10100], 4112, 16), ([4300], 4112, 48), ([100, 4200], 4112, 144),
          ([7900], 2064, 272), ([5100], 4096, 96)]


@pytest.mark.parametrize("act", [False, True])
@pytest.mark.parametrize("sizes,N,K", ROUNDS)
def test_matmul_rounds(sizes, N, K, act):
    products(sum(sizes), N, K, sizes, len(sizes), act, K > 100, seed=N)


def test_matmul_one_weight_past_32_bits():
    """N * K over 4 GB: the last channels, for few rows and for many."""
    N, K = 69_648, 65_536
    wq = torch.zeros(1, N, K, dtype=torch.int8, device="cuda")
    wq[0, -16:] = torch.randint(-127, 128, (16, K), dtype=torch.int8, device="cuda")
    wq[0, N // 2 - 16:N // 2] = torch.randint(-127, 128, (16, K), dtype=torch.int8, device="cuda")
    w = np.concatenate([wq[0, N // 2 - 16:N // 2].cpu().numpy(), wq[0, -16:].cpu().numpy()])[None]
    for M in (2, 70, 400):
        xq = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda")
        xs, ws = torch.rand(M, device="cuda") * 1e-3, torch.rand(1, N, device="cuda") * 1e-3
        s = torch.cat([ws[:, N // 2 - 16:N // 2], ws[:, -16:]], 1).cpu().numpy()
        for act in (False, True):
            y, st = torch.ones(M, N // 2 if act else N, device="cuda"), status()
            uep.ultraep_expert_matmul(xq, xs, M, wq, ws, 1, N, K, torch.tensor([0, M], device="cuda"), None, 1, act, y, st)
            want, rel = p64.expert_matmul(xq.cpu().numpy(), xs.cpu().numpy(), w, s, [0, M], None, act)
            got = (y[:, -16:] if act else torch.cat([y[:, N // 2 - 16:N // 2], y[:, -16:]], 1)).double().cpu().numpy()
            assert (np.abs(got - want) <= rel * np.abs(want) + 1e-37).all()
            assert not y[:, :N // 2 - 16].any() and int(st.item()) == 0


def test_matmul_part_of_the_blocks():
    """Blocks that begin and end inside the rows."""
    products(300, 80, 96, [40, 0, 100], 3, False, False, start=37)


@pytest.mark.parametrize("M", [4, 300])
def test_matmul_largest_sums(M):
    """127 * 127 * K at the longest K: the sum just fits 32 bits."""
    products(M, 16, 1 << 16, [M], 1, False, True, extreme=True)


def test_matmul_part_of_many_rows():
    products(6000, 1040, 80, [1500, 0, 2100], 3, True, False, start=301)


@pytest.mark.parametrize("M", [3, 400])
def test_matmul_bad_blocks(M):
    """Out of order, out of range, or without a weight: reported, and nothing written."""
    N, K = 64, 64
    xq, wq = torch.ones(M, K, dtype=torch.int8, device="cuda"), torch.ones(2, N, K, dtype=torch.int8, device="cuda")
    xs, ws = torch.ones(M, device="cuda"), torch.ones(2, N, device="cuda")
    for off, of in [([0, 2, 1], None), ([0, 1, M + 1], None), ([-1, 1, 2], None), ([0, 1, 2], [0, 2]),
                    ([0, 1, 2], [-1, 1]), ([0, 1 << 40, 1 << 41], None)]:
        y, st = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), status()
        uep.ultraep_expert_matmul(xq, xs, M, wq, ws, 2, N, K, dev(np.array(off, np.int64)),
                                  None if of is None else dev(np.array(of, np.int32)), 2, False, y, st)
        assert int(st.item()) == uep.ULTRAEP_EDATA and not y.any()
    off = np.full(201, M, np.int64)  # a bad block among several runs of 64
    off[:101:2], off[1:101:2] = 0, M
    y, st = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), status()
    uep.ultraep_expert_matmul(xq, xs, M, wq, ws, 2, N, K, dev(off), dev(np.zeros(200, np.int32)), 200, False, y, st)
    assert int(st.item()) == uep.ULTRAEP_EDATA and not y.any()
    y, st = torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), status()
    uep.ultraep_expert_matmul(xq, xs, M, wq, ws, 2, N, K, dev(np.array([0, 2, 2], np.int64)),
                              dev(np.array([1, -1], np.int32)), 2, False, y, st)
    assert int(st.item()) == 0 and (y[:2] == K).all()  # an empty block needs no weight


def test_matmul_scales_carry_nan_and_infinity():
    xq, wq = torch.ones(3, 32, dtype=torch.int8, device="cuda"), torch.ones(1, 16, 32, dtype=torch.int8, device="cuda")
    xs = torch.tensor([float("nan"), float("inf"), 1.0], device="cuda")
    for act in (False, True):
        y, st = torch.empty(3, 8 if act else 16, dtype=torch.bfloat16, device="cuda"), status()
        uep.ultraep_expert_matmul(xq, xs, 3, wq, torch.ones(1, 16, device="cuda"), 1, 16, 32,
                                  torch.tensor([0, 3], device="cuda"), None, 1, act, y, st)
        assert (y[0].view(torch.int16) == 0x7FC0).all() and torch.isinf(y[1]).all() and torch.isfinite(y[2]).all()


@pytest.mark.parametrize("M,N", [(1_100_003, 16), (300_000, 8192)])
def test_matmul_offsets_past_32_bits(M, N):
    """xq, and y, of over 4 GB: the last rows."""
    K = 4096 if N == 16 else 16
    xq = torch.zeros(M, K, dtype=torch.int8, device="cuda")
    xq[-5:] = torch.randint(-127, 128, (5, K), dtype=torch.int8, device="cuda")
    wq = torch.randint(-127, 128, (1, N, K), dtype=torch.int8, device="cuda")
    xs, ws = torch.rand(M, device="cuda"), torch.rand(1, N, device="cuda")
    y, st = torch.ones(M, N, dtype=torch.bfloat16, device="cuda"), status()
    uep.ultraep_expert_matmul(xq, xs, M, wq, ws, 1, N, K, torch.tensor([0, M], device="cuda"), None, 1, False, y, st)
    want, rel = p64.expert_matmul(xq[-5:].cpu().numpy(), xs[-5:].cpu().numpy(), wq.cpu().numpy(), ws.cpu().numpy(),
                                  [0, 5], None, False)
    got = y[-5:].double().cpu().numpy()
    assert (np.abs(got - want) <= (rel + 1.01 * p64.U16) * np.abs(want)).all()
    assert not y[:-5].any() and int(st.item()) == 0


def test_matmul_weights_past_32_bits():
    n_w, N, K = 5, 16384, 65536
    wq = torch.zeros(n_w, N, K, dtype=torch.int8, device="cuda")
    wq[-1, -16:] = torch.randint(-127, 128, (16, K), dtype=torch.int8, device="cuda")
    for M in (2, 200):
        xq = torch.randint(-127, 128, (M, K), dtype=torch.int8, device="cuda")
        xs, ws = torch.rand(M, device="cuda"), torch.rand(n_w, N, device="cuda")
        y, st = torch.ones(M, N, device="cuda"), status()
        uep.ultraep_expert_matmul(xq, xs, M, wq, ws, n_w, N, K, torch.tensor([0, M], device="cuda"),
                                  torch.tensor([n_w - 1], dtype=I32, device="cuda"), 1, False, y, st)
        want, rel = p64.expert_matmul(xq.cpu().numpy(), xs.cpu().numpy(), wq[-1:, -16:].cpu().numpy(),
                                      ws[-1:, -16:].cpu().numpy(), [0, M], None, False)
        got = y[:, -16:].double().cpu().numpy()
        assert (np.abs(got - want) <= rel * np.abs(want)).all()
        assert not y[:, :-16].any() and int(st.item()) == 0


# ---------------------------------------------------------------- combine_grad

def layout(rng, T, k, masked, n_rows):
    """Slots in a random order of rows, a share of them masked."""
    on = rng.random(T * k) >= masked
    n = int(on.sum())
    rows = np.full(T * k, -1, np.int32)
    rows[on] = rng.permutation(n)
    return rows, n


@pytest.mark.parametrize("T,k,H,masked,extra", [
    (1, 1, 8, 0, 0), (1, 8, 7168, 0, 0), (7, 3, 24, 0.3, 5), (50, 8, 520, 0.2, 0), (33, 12, 2056, 0.1, 3),
    (20, 64, 136, 0.5, 0), (300, 2, 256, 0, 0), (9, 9, 4104, 0, 1), (5, 6, 2880, 1.0, 0), (64, 8, 12288, 0.05, 0),
    (3, 17, 16392, 0.2, 40)])
def test_combine_grad(T, k, H, masked, extra):
    rng = np.random.default_rng(T * H)
    n_rows = T * k + extra
    rows, n = layout(rng, T, k, masked, n_rows)
    dout = p64.bf16(rng.standard_normal((T, H)).astype(np.float32))
    y = p64.bf16(rng.standard_normal((n_rows, H)).astype(np.float32))
    gate = rng.random((T, k)).astype(np.float32)
    dy = torch.full((n_rows * H + 8,), 99, dtype=torch.int16, device="cuda")
    dg = torch.full((T * k + 4,), 9., device="cuda")
    st = status()
    uep.ultraep_combine_grad(dev(p64.bf16_bits(dout).view(np.int16)), dev(p64.bf16_bits(y).view(np.int16)), n_rows,
                             dev(gate), dev(rows), T, k, H, torch.tensor([n], device="cuda"), dy, dg, st)
    assert int(st.item()) == 0
    got = dy[:n_rows * H].cpu().numpy().view(np.uint16).reshape(n_rows, H)
    want = np.zeros((n_rows, H), np.uint16)
    slots = np.flatnonzero(rows >= 0)
    want[rows[slots]] = p64.bf16_bits(gate.reshape(-1)[slots, None] * dout[slots // k])
    assert np.array_equal(got, want)
    assert (dy[n_rows * H:] == 99).all() and (dg[T * k:] == 9).all()
    g = dg[:T * k].cpu().numpy()
    assert (g[rows < 0] == 0).all()
    a, b = dout[slots // k].astype(np.float64), y[rows[slots]].astype(np.float64)
    assert (np.abs(g[slots] - (a * b).sum(1)) <= (H + 1) * p64.U32 * np.abs(a * b).sum(1)).all()


@pytest.mark.parametrize("T,H", [(256, 4096), (256, 4104), (257, 4104), (40, 512), (40, 520), (700, 8)])
def test_combine_grad_at_each_workgroup_size(T, H):
    test_combine_grad(T, 3, H, 0.2, 2)


def test_combine_grad_is_the_gradient_of_the_combine():
    """Of the objective sum dout * combine(y, gate), linear in y and in gate: the
    objective's change along random directions, in 64 bits."""
    rng = np.random.default_rng(1)
    T, k, H = 12, 4, 64
    rows, n = layout(rng, T, k, 0.2, T * k)
    dout, y = (p64.bf16(rng.standard_normal(s).astype(np.float32)) for s in ((T, H), (T * k, H)))
    gate = rng.random((T, k)).astype(np.float32)
    dy, dg, st = (torch.empty(T * k, H, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, device="cuda"), status())
    uep.ultraep_combine_grad(dev(p64.bf16_bits(dout).view(np.int16)), dev(p64.bf16_bits(y).view(np.int16)), T * k,
                             dev(gate), dev(rows), T, k, H, torch.tensor([n], device="cuda"), dy, dg, st)

    def objective(y, gate):
        out = np.zeros((T, H))
        for s in np.flatnonzero(rows >= 0):
            out[s // k] += gate.reshape(-1)[s] * y[rows[s]]
        return (out * dout).sum()
    y64, g64 = y.astype(np.float64), gate.astype(np.float64)
    for _ in range(5):
        ey, eg = rng.standard_normal(y.shape), rng.standard_normal(gate.shape)
        gy = dy.double().cpu().numpy()
        along = objective(y64 + ey, g64) - objective(y64, g64)
        assert abs((gy * ey).sum() - along) <= 1.01 * p64.U16 * (np.abs(gy * ey)).sum() + 1e-9
        gg = dg.double().cpu().numpy()
        along = objective(y64, g64 + eg) - objective(y64, g64)
        size = np.zeros((T * k,))
        on = np.flatnonzero(rows >= 0)
        size[on] = (np.abs(dout[on // k]) * np.abs(y[rows[on]])).sum(1)
        assert abs((gg * eg).sum() - along) <= (H + 1) * p64.U32 * (size * np.abs(eg).reshape(-1)).sum() + 1e-9


def test_combine_grad_data_errors():
    T, k, H = 6, 2, 16
    dout, y = torch.ones(T, H, dtype=torch.bfloat16, device="cuda"), torch.ones(12, H, dtype=torch.bfloat16, device="cuda")
    gate = torch.ones(T, k, device="cuda")

    def call(rows, n):
        dy, dg, st = torch.full_like(y, 3), torch.full_like(gate, 3), status()
        uep.ultraep_combine_grad(dout, y, 12, gate, torch.tensor(rows, dtype=I32, device="cuda"), T, k, H,
                                 torch.tensor([n], device="cuda"), dy, dg, st)
        return dy, dg, int(st.item())
    ok = list(range(12))
    assert call(ok, 12)[2] == 0
    for bad in (-2, 12, 1 << 30):
        rows = ok[:]
        rows[5] = bad
        dy, dg, st = call(rows, 12)
        assert st == uep.ULTRAEP_EDATA and float(dg.view(-1)[5]) == 0 and float(dg.view(-1)[4]) == H
    dy, dg, st = call(ok, 9)  # rows past the routed ones
    assert st == uep.ULTRAEP_EDATA and (dy[9:] == 0).all()
    for n in (-1, 13):
        dy, dg, st = call(ok, n)
        assert st == uep.ULTRAEP_EDATA and (dy == 3).all() and (dg == 0).all()


def test_combine_grad_no_tokens_and_nan():
    dy, st = torch.full((5, 8), 3, dtype=torch.bfloat16, device="cuda"), status()
    y = torch.ones_like(dy)
    uep.ultraep_combine_grad(None, y, 5, None, None, 0, 2, 8, torch.tensor([0], device="cuda"), dy, None, st)
    assert (dy == 0).all() and int(st.item()) == 0
    dout = torch.full((1, 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    dg = torch.empty(1, 2, device="cuda")
    uep.ultraep_combine_grad(dout, y, 5, torch.ones(1, 2, device="cuda"), torch.tensor([1, -1], dtype=I32, device="cuda"),
                             1, 2, 8, torch.tensor([2], device="cuda"), dy, dg, st)
    assert (dy[1].view(torch.int16) == 0x7FC0).all() and torch.isnan(dg[0, 0]) and float(dg[0, 1]) == 0


def test_combine_grad_offsets_past_32_bits():
    T, k, H = 40_000, 8, 8192
    n = T * k
    dout = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(n, H, dtype=torch.bfloat16, device="cuda")
    dout[-1], y[-8:] = 1.5, 2.0
    gate = torch.full((T, k), 0.5, device="cuda")
    dy, dg, st = torch.ones_like(y), torch.empty(T, k, device="cuda"), status()
    uep.ultraep_combine_grad(dout, y, n, gate, torch.arange(n, dtype=I32, device="cuda"), T, k, H,
                             torch.tensor([n], device="cuda"), dy, dg, st)
    assert (dy[-8:] == 0.75).all() and not dy[:-8].any()
    assert (dg[-1] == 3 * H).all() and not dg[:-1].any() and int(st.item()) == 0


# -------------------------------------------------------- streams, graphs, types

def test_other_stream_and_equal_bits():
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(300, 256, device="cuda", generator=g).to(torch.bfloat16)
    w = torch.randn(4 * 128, 256, device="cuda", generator=g).to(torch.bfloat16)
    off, st = torch.tensor([0, 100, 100, 290, 300], device="cuda"), status()
    outs = []
    for s in (None, torch.cuda.Stream()):
        if s is not None:
            s.wait_stream(torch.cuda.current_stream())
        q, xs = torch.empty(300, 256, dtype=torch.int8, device="cuda"), torch.empty(300, device="cuda")
        wq, ws = torch.empty(512, 256, dtype=torch.int8, device="cuda"), torch.empty(512, device="cuda")
        y = torch.empty(300, 64, dtype=torch.bfloat16, device="cuda")
        torch.cuda.synchronize()
        uep.ultraep_quant_rows(x, 300, 256, 256, q, 256, xs, stream=s)
        uep.ultraep_quant_rows(w, 512, 256, 256, wq, 256, ws, stream=s)
        uep.ultraep_expert_matmul(q, xs, 300, wq, ws, 4, 128, 256, off, None, 4, True, y, st, stream=s)
        torch.cuda.synchronize()
        outs.append((q, xs, y))
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and int(st.item()) == 0


@pytest.mark.parametrize("M", [8, 400])
def test_graph_replay(M):
    K, N, k = 256, 128, 2
    x, w = torch.empty(M, K, device="cuda"), torch.randn(2 * N, K, device="cuda")
    q, xs = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    wq, ws = torch.empty(2 * N, K, dtype=torch.int8, device="cuda"), torch.empty(2 * N, device="cuda")
    y, st = torch.empty(M, N, dtype=torch.bfloat16, device="cuda"), status()
    off = torch.tensor([0, M // 3, M], device="cuda")
    dy, dg = torch.empty_like(y), torch.empty(M // k, k, device="cuda")
    gate, rows = torch.rand(M // k, k, device="cuda"), torch.randperm(M, device="cuda").to(I32)
    dout, n = torch.randn(M // k, N, device="cuda").to(torch.bfloat16), torch.tensor([M], device="cuda")
    uep.ultraep_quant_rows(w, 2 * N, K, K, wq, K, ws)

    def step():
        uep.ultraep_quant_rows(x, M, K, K, q, K, xs)
        uep.ultraep_expert_matmul(q, xs, M, wq, ws, 2, N, K, off, None, 2, False, y, st)
        uep.ultraep_combine_grad(dout, y, M, gate, rows, M // k, k, N, n, dy, dg, st)
    x.normal_()
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        x.normal_()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (q, xs, y, dy, dg)]
        for t in (q, xs, y, dy, dg):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (q, xs, y, dy, dg)))
    assert int(st.item()) == 0
