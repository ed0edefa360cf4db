"""The experts' operators at their limits: over 2^31 - 1 rows, all zero but for some from one end
to the other (what those give, and that the others give zeros), and over 2^20 channels or
elements of a row (2^18 in 8 bits).  Needs an MI355X."""
import pytest
import torch

from test_gpu_expert_products import status

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

M = (1 << 31) - 1
AT = [0, 63, 64, (1 << 30) - 1, (1 << 30) + 5, M - 257, M - 256, M - 65, M - 64, M - 1]
BF16, U8 = torch.bfloat16, torch.uint8


@pytest.fixture(autouse=True)
def memory():
    """What a test took is given back: tens of GB."""
    yield
    torch.cuda.empty_cache()


def integers(g, *shape):
    return torch.randint(-3, 4, shape, device="cuda", generator=g).to(BF16)


def others_are_zero(t):
    """Rows that are not among AT; which are cleared."""
    t[AT] = 0
    return all(not t[lo:lo + (1 << 27)].view(torch.int64).any() for lo in range(0, M, 1 << 27))


@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("sizes", [[M], [(1 << 30) + 3, 0, M - (1 << 30) - 3]])
def test_bf16_products(trans, sizes):
    """Integers of at most 3: every sum is exact."""
    N = K = 8
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w = torch.zeros(M, K, dtype=BF16, device="cuda"), integers(g, 1, N, K)
    x[AT] = integers(g, len(AT), K)
    y = torch.full((M, N), 3.0, dtype=BF16, device="cuda")
    st, n = status(), len(sizes)
    off = torch.tensor([0] + sizes, device="cuda").cumsum(0)
    uep.ultraep_expert_matmul_bf16(x, M, w, 1, N * K, N, K, trans, off, torch.zeros(n, dtype=torch.int32, device="cuda"), n,
                                   uep.ULTRAEP_NO_ACT, None, y, st)
    assert int(st.item()) == 0
    assert torch.equal(y[AT].double(), x[AT].double() @ (w[0] if trans else w[0].t().contiguous()).double())
    assert others_are_zero(y)


def test_quantised_and_multiplied_in_8_bits():
    N, K = 8, 16
    g = torch.Generator(device="cuda").manual_seed(6)
    x, w = torch.zeros(M, K, dtype=BF16, device="cuda"), integers(g, N, K)
    x[AT] = integers(g, len(AT), K)
    xq, xs = torch.full((M, K), 77, dtype=U8, device="cuda"), torch.full((M, 4), 77, dtype=U8, device="cuda")
    wq, ws = torch.empty(N, K, dtype=U8, device="cuda"), torch.empty(N, 4, dtype=U8, device="cuda")
    uep.ultraep_quant_blocks(x, M, K, K, xq, K, xs)
    uep.ultraep_quant_blocks(w, N, K, K, wq, K, ws)
    want = x[AT].double() @ w.double().t().contiguous()
    del x
    y, st = torch.full((M, N), 3.0, dtype=BF16, device="cuda"), status()
    uep.ultraep_expert_matmul_fp8(xq, xs, M, wq, ws, 1, N, K, torch.tensor([0, M], device="cuda"), None, 1, 0, y, st)
    assert int(st.item()) == 0 and torch.equal(y[AT].double(), want)
    assert others_are_zero(y) and others_are_zero(xq)
    xs[AT] = 0
    assert not xs.view(torch.int32).any()  # (a row of zeros has the least scale, whose byte is 0)


@pytest.mark.parametrize("rows", [1, 70, 300])
@pytest.mark.parametrize("N,K", [(1 << 20, 64), (48, 1 << 20), (1 << 20, 72)])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("act", [0, 1])
def test_the_widest_bf16_products(rows, N, K, trans, act):
    """Integers: sums below 2^24, exact (SwiGLU: what it keeps)."""
    g = torch.Generator(device="cuda").manual_seed(7)
    x, w = integers(g, rows, K), integers(g, *((K, N) if trans else (N, K)))
    y = torch.empty(rows, N // 2 if act else N, device="cuda")
    pre = torch.empty(rows, N, dtype=BF16, device="cuda") if act else None
    st = status()
    uep.ultraep_expert_matmul_bf16(x, rows, w, 1, N * K, N, K, trans, torch.tensor([0, rows], device="cuda"), None, 1, act, pre,
                                   y, st)
    assert int(st.item()) == 0
    want = x.float() @ (w if trans else w.t().contiguous()).float()
    assert torch.equal(pre, want.to(BF16)) if act else torch.equal(y, want)


@pytest.mark.parametrize("rows", [1, 130])
@pytest.mark.parametrize("N,K", [(1 << 20, 64), (48, 1 << 20)])
@pytest.mark.parametrize("swap", [False, True])
def test_the_widest_weight_gradients(rows, N, K, swap):
    N, K = (K, N) if swap else (N, K)
    g = torch.Generator(device="cuda").manual_seed(8)
    dy, x = integers(g, rows, N), integers(g, rows, K)
    dw, st = torch.empty(N, K, device="cuda"), status()
    uep.ultraep_expert_weight_grad(dy, x, rows, N, K, torch.tensor([0, rows], device="cuda"), None, 1, 1, N * K, False, dw, None,
                                   st)
    assert int(st.item()) == 0 and torch.equal(dw, dy.float().t().contiguous() @ x.float())


@pytest.mark.parametrize("rows", [1, 70, 300])
@pytest.mark.parametrize("N,K", [(1 << 20, 528), (48, 1 << 18)])
def test_the_widest_8_bit_products(rows, N, K):
    g = torch.Generator(device="cuda").manual_seed(9)
    x, w = integers(g, rows, K), integers(g, N, K)
    (xq, xs), (wq, ws) = ((torch.empty(t.shape, dtype=U8, device="cuda"),
                           torch.empty(t.shape[0], uep.scale_pitch(K), dtype=U8, device="cuda")) for t in (x, w))
    for t, q, s in ((x, xq, xs), (w, wq, ws)):
        uep.ultraep_quant_blocks(t, t.shape[0], K, K, q, K, s)
    y, st = torch.empty(rows, N, dtype=BF16, device="cuda"), status()
    uep.ultraep_expert_matmul_fp8(xq, xs, rows, wq, ws, 1, N, K, torch.tensor([0, rows], device="cuda"), None, 1, 0, y, st)
    assert int(st.item()) == 0
    assert torch.equal(y, (x.float() @ w.float().t().contiguous()).to(BF16))
