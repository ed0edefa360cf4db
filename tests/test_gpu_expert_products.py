"""The experts' products in bf16 and in 8-bit floating point, the weights' gradient
and the block quantisation on the GPU, against the plain 64-bit implementations
and within the bounds that plain_experts derives.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import plain64 as p64
import plain_experts as pe

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep
    ACTS = {"none": uep.ULTRAEP_NO_ACT, "swiglu": uep.ULTRAEP_SWIGLU, "swiglu_grad": uep.ULTRAEP_SWIGLU_GRAD}

I32, I64, F32, BF16, U8 = torch.int32, torch.int64, torch.float32, torch.bfloat16, torch.uint8


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def dev16(a):
    return dev(p64.bf16_bits(a).view(np.int16))


def status():
    return torch.zeros(1, dtype=I32, device="cuda")


def layout(sizes, start, tail):
    off = start + np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    return off, int(off[-1]) + tail


def normal(rng, *shape):
    return p64.bf16(rng.standard_normal(shape).astype(np.float32))


def same_where_defined(got, want, err):
    bad = ~(np.abs(got - want) <= err)
    bad &= ~np.isnan(want)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:5].tolist(), got[bad][:5], want[bad][:5], err[bad][:5])


# --------------------------------------------------------------- bf16 products

def bf16_product(sizes, N, K, trans, act, f32, of=None, n_w=None, start=0, tail=0, gap=0, keep=True, seed=0, spoil=None):
    rng = np.random.default_rng(seed)
    off, M = layout(sizes, start, tail)
    n_w = n_w or len(sizes)
    x, w = normal(rng, M, K), normal(rng, n_w, *((K, N) if trans else (N, K)))
    pre = normal(rng, M, 2 * N) * 2 if act == "swiglu_grad" else None
    if spoil:
        spoil(x, w, pre)
    blob = np.full((n_w, N * K + gap), np.nan, np.float32)
    blob[:, :N * K] = w.reshape(n_w, -1)
    width = {"none": N, "swiglu": N // 2, "swiglu_grad": 2 * N}[act]
    y = torch.full((M, width), 3.0, dtype=F32 if f32 else BF16, device="cuda")
    p = dev16(pre) if pre is not None else None
    if act == "swiglu" and keep:
        p = torch.full((M, N), 5.0, dtype=BF16, device="cuda")
    st = status()
    uep.ultraep_expert_matmul_bf16(dev16(x), M, dev16(blob), n_w, N * K + gap, N, K, trans, dev(off),
                                   None if of is None else dev(np.array(of, np.int32)), len(sizes), ACTS[act], p, y, st)
    assert int(st.item()) == 0
    want, err, v, dv = pe.product(x.astype(np.float64), w.astype(np.float64), off, of, act, trans,
                                  None if pre is None else pre.astype(np.float64))
    got = y.double().cpu().numpy()
    inside = np.zeros(M, bool)
    inside[off[0]:off[-1]] = True
    assert (got[~inside] == 3).all()  # rows outside the blocks are left alone
    if act == "swiglu" and keep:
        kept = p.double().cpu().numpy()
        assert (kept[~inside] == 5).all()
        return got, want, pe.rounded(want, err, f32), kept, v, pe.rounded(v, dv, False), inside
    return got, want, pe.rounded(want, err, f32), None, None, None, inside


def check_bf16(*args, **kw):
    got, want, err, kept, v, dv, inside = bf16_product(*args, **kw)
    assert np.isfinite(got).all()
    same_where_defined(got[inside], want[inside], err[inside])
    if kept is not None:
        same_where_defined(kept[inside], v[inside], dv[inside])


SHAPES = [  # sizes, N, K
    ([1], 16, 8), ([1], 64, 4096), ([0, 3, 0], 48, 24), ([65, 0, 63, 1], 96, 72), ([130, 7], 272, 136),
    ([5, 64, 128, 200], 144, 520), ([257], 528, 64), ([300, 300], 320, 200), ([16, 16, 16, 16], 1040, 2056)]


@pytest.mark.parametrize("sizes,N,K", SHAPES)
@pytest.mark.parametrize("act", ["none", "swiglu", "swiglu_grad"])
@pytest.mark.parametrize("trans", [False, True])
def test_bf16_products(sizes, N, K, trans, act):
    check_bf16(sizes, N, K, trans, act, f32=False)


@pytest.mark.parametrize("act", ["none", "swiglu", "swiglu_grad"])
@pytest.mark.parametrize("trans", [False, True])
@pytest.mark.parametrize("sizes,N,K", [([70, 3], 80, 40), ([1], 32, 520), ([300, 41], 336, 136)])
def test_bf16_products_fp32_results(sizes, N, K, trans, act):
    check_bf16(sizes, N, K, trans, act, f32=True, gap=N * 8, start=2, tail=3)


@pytest.mark.parametrize("trans", [False, True])
def test_bf16_products_of_shared_weights_and_spare_rows(trans):
    check_bf16([40, 0, 33, 90], 64, 96, trans, "none", False, of=[2, 7, 0, 2], n_w=3, start=5, tail=9, gap=24)


def test_swiglu_without_kept_channels():
    check_bf16([40, 100], 64, 96, False, "swiglu", False, keep=False)


@pytest.mark.parametrize("trans", [False, True])
def test_bf16_products_of_many_blocks(trans):
    rng = np.random.default_rng(1)
    sizes = rng.integers(0, 4, 2048)
    sizes[[70, 900, 2047]] = [150, 0, 65]
    of = rng.integers(0, 5, 2048)
    of[sizes == 0] = -7  # an empty block needs no weight
    check_bf16(sizes.tolist(), 32, 40, trans, "none", False, of=of.tolist(), n_w=5)


TILES = [  # every choice of tiles: one to four blocks of a few rows to many, wide and narrow
    ([1200], 1032, 264), ([520, 700], 768, 136), ([90] * 24, 776, 72), ([48] * 20, 1040, 328), ([20] * 9, 528, 1160),
    ([3000], 264, 72), ([33] * 64, 520, 200), ([8] * 40, 1024, 4104), ([24] * 30, 1040, 4104), ([40] * 30, 1040, 4104)]


def shared(sizes):
    """Many blocks over five weights."""
    return dict(of=[g * 3 % 5 for g in range(len(sizes))], n_w=5) if len(sizes) > 5 else {}


@pytest.mark.parametrize("sizes,N,K", TILES)
@pytest.mark.parametrize("trans,act", [(False, "none"), (True, "none"), (False, "swiglu"), (True, "swiglu_grad")])
def test_bf16_products_over_the_tile_shapes(sizes, N, K, trans, act):
    if act == "swiglu":
        N = N // 16 * 16
    check_bf16(sizes, N, K, trans, act, f32=False, **shared(sizes))


MANY = [  # enough tiles for the largest, whole rounds of them and not, and many blocks of middling rows
    ([4096], 4088, 72), ([2000, 2230], 4088, 72), ([2040], 4096, 72), ([2040], 2040, 136), ([60] * 60, 264, 2056),
    ([40] * 40, 264, 4104), ([50] * 50, 128, 136), ([50] * 50, 128, 4112)]


@pytest.mark.parametrize("sizes,N,K", MANY)
@pytest.mark.parametrize("trans,act", [(False, "none"), (True, "none"), (False, "swiglu"), (True, "swiglu"), (False, "swiglu_grad"), (True, "swiglu_grad")])
def test_bf16_products_of_many_tiles(sizes, N, K, trans, act):
    check_bf16(sizes, N // 16 * 16 if act == "swiglu" else N, K, trans, act, f32=False, **shared(sizes))


@pytest.mark.parametrize("sizes,N,K", MANY[1:3] + MANY[4:6])
@pytest.mark.parametrize("trans,act", [(True, "none"), (False, "swiglu")])
def test_bf16_products_of_many_tiles_fp32_results(sizes, N, K, trans, act):
    check_bf16(sizes, N // 16 * 16, K, trans, act, f32=True, **shared(sizes))


@pytest.mark.parametrize("trans", [False, True])
def test_bf16_products_of_other_numbers(trans):
    """Infinities and NaN stay in their row, channel and block."""
    def spoil(x, w, pre):
        x[3, 5], x[10, 0], x[64, 39] = np.nan, np.inf, -np.inf
        if trans:
            w[1, 2, 9], w[1, 39, 0] = np.inf, np.nan
        else:
            w[1, 9, 2], w[1, 0, 39] = np.inf, np.nan
    got, want, err, _, _, _, _ = bf16_product([30, 50], 24, 40, trans, "none", True, spoil=spoil)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert inf.any() and np.array_equal(got[inf], want[inf])
    fine = np.isfinite(want)
    assert (np.abs(got - want) <= err)[fine].all()


@pytest.mark.parametrize("K", [8, 24, 56, 72, 120, 136])
@pytest.mark.parametrize("trans", [False, True])
def test_bf16_products_read_nothing_beyond_a_row(trans, K):
    """The row after a block's last and the weight after a block's hold NaN."""
    def spoil(x, w, pre):
        x[:2] = x[-3:] = np.nan
        w[0] = w[2] = np.nan
    got, want, err, _, _, _, inside = bf16_product([21], 40, K, trans, "none", True, of=[1], n_w=3, start=2, tail=3,
                                                   spoil=spoil)
    assert np.isfinite(got).all()
    same_where_defined(got[inside], want[inside], err[inside])


def test_swiglu_of_large_and_small_gates():
    """Gates from -200 to 200, and infinite ones: silu(-inf) is 0 * inf in neither half."""
    M, N, K = 33, 32, 8
    x = np.zeros((M, K), np.float32)
    x[:, 0] = np.linspace(-200, 200, M)
    x[:, 1] = 1.0
    x = p64.bf16(x)
    w = np.zeros((1, N, K), np.float32)
    w[0, :16, 0] = 1.0
    w[0, 16:, 1] = 2.0
    y = torch.empty(M, 16, dtype=F32, device="cuda")
    uep.ultraep_expert_matmul_bf16(dev16(x), M, dev16(w), 1, N * K, N, K, False, dev(np.array([0, M])), None, 1,
                                   uep.ULTRAEP_SWIGLU, None, y, status())
    a = x[:, :1].astype(np.float64)
    want = np.repeat(2 * pe.silu(a), 16, axis=1)
    same_where_defined(y.double().cpu().numpy(), want, (16 + 3 * np.abs(a)) * p64.U32 * np.abs(want) + 3 * pe.TINY)
    pre = np.zeros((M, 2 * N), np.float32)
    pre[:, :N], pre[:, N:] = x[:, :1], 3.0
    dy = torch.empty(M, 2 * N, dtype=F32, device="cuda")
    one = np.zeros((M, K), np.float32)
    one[:, 0] = 1.0
    w1 = np.zeros((1, N, K), np.float32)
    w1[:, :, 0] = 1.0
    uep.ultraep_expert_matmul_bf16(dev16(one), M, dev16(w1), 1, N * K, N, K, False, dev(np.array([0, M])), None, 1,
                                   uep.ULTRAEP_SWIGLU_GRAD, dev16(pre), dy, status())
    want, err = pe.activate(np.ones((M, N)), np.zeros((M, N)), "swiglu_grad", pre.astype(np.float64))
    same_where_defined(dy.double().cpu().numpy(), want, err + p64.U32 * np.abs(want) + 3 * pe.TINY)


def test_swiglu_gradient_in_place():
    rng = np.random.default_rng(4)
    M, N, K = 200, 144, 72
    x, w, pre = (dev16(normal(rng, *s)) for s in ((M, K), (2, K, N), (M, 2 * N)))
    off, y = dev(np.array([0, 77, M])), torch.empty(M, 2 * N, dtype=BF16, device="cuda")
    args = (x, M, w, 2, N * K, N, K, True, off, None, 2, uep.ULTRAEP_SWIGLU_GRAD)
    uep.ultraep_expert_matmul_bf16(*args, pre, y, status())
    uep.ultraep_expert_matmul_bf16(*args, pre, pre, status())
    assert torch.equal(pre.view(BF16), y)


BAD_LISTS = [([0, 5, 3, 20], None), ([-1, 5, 8, 20], None), ([0, 5, 8, 21], None), ([0, 5, 8, 20], [0, 3, 1]),
             ([0, 5, 8, 20], [0, -1, 1]), ([4, 2, 8, 20], None)]


@pytest.mark.parametrize("off,of", BAD_LISTS)
def test_unsound_blocks_write_nothing(off, of):
    M, N, K, n_w = 20, 32, 48, 3
    x, w = torch.ones(M, K, dtype=BF16, device="cuda"), torch.ones(n_w, N, K, dtype=BF16, device="cuda")
    o, b = dev(np.array(off, np.int64)), None if of is None else dev(np.array(of, np.int32))
    y, pre = torch.full((M, N // 2), 3.0, device="cuda"), torch.full((M, N), 3.0, dtype=BF16, device="cuda")
    st = status()
    uep.ultraep_expert_matmul_bf16(x, M, w, n_w, N * K, N, K, False, o, b, 3, uep.ULTRAEP_SWIGLU, pre, y, st)
    assert int(st.item()) == uep.ULTRAEP_EDATA and (y == 3).all() and (pre == 3).all()
    st = status()
    dw = torch.full((n_w, N, K), 3.0, device="cuda")
    for ws in (None, torch.empty(uep.ultraep_expert_weight_grad_ws_bytes(M, N, K, n_w), dtype=U8, device="cuda")):
        uep.ultraep_expert_weight_grad(torch.ones(M, N, dtype=BF16, device="cuda"), x, M, N, K, o, b, 3, n_w, N * K, False,
                                       dw, ws, st)
        assert int(st.item()) == uep.ULTRAEP_EDATA and (dw == 3).all()
    st = status()
    y = torch.full((M, N), 3.0, device="cuda")
    uep.ultraep_expert_matmul_fp8(torch.zeros(M, K, dtype=U8, device="cuda"), torch.zeros(M, 4, dtype=U8, device="cuda"), M,
                                  torch.zeros(n_w, N, K, dtype=U8, device="cuda"),
                                  torch.zeros(n_w, N, 4, dtype=U8, device="cuda"), n_w, N, K, o, b, 3, 0, y, st)
    assert int(st.item()) == uep.ULTRAEP_EDATA and (y == 3).all()


@pytest.mark.parametrize("trans", [False, True])
def test_bf16_products_offsets_past_32_bits(trans):
    """Weights of over 4 GiB, rows of over 4 GiB."""
    n_w, N, K = 5, 16384, 32768
    w = torch.zeros(n_w, N * K, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    w[4].normal_(generator=g)
    x = torch.randn(3, K, device="cuda", generator=g).to(BF16)
    y, st = torch.empty(3, N, device="cuda"), status()
    uep.ultraep_expert_matmul_bf16(x, 3, w, n_w, N * K, N, K, trans, dev(np.array([0, 1, 3])),
                                   dev(np.array([4, 4], np.int32)), 2, 0, None, y, st)
    v = w[4].view(K, N) if trans else w[4].view(N, K).t()
    xd = x.double()
    want, mag = torch.zeros(3, N, dtype=torch.float64, device="cuda"), torch.zeros(3, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 4096):
        part = v[k:k + 4096].double().contiguous()
        want += xd[:, k:k + 4096] @ part
        mag += xd[:, k:k + 4096].abs() @ part.abs()
    assert int(st.item()) == 0 and ((y - want).abs() <= 2 * K * p64.U32 * mag + p64.U32 * want.abs()).all()
    del w, v
    M, N, K = 300_000, 8192, 64
    w = torch.randn(1, N * K, device="cuda", generator=g).to(BF16)
    x = torch.zeros(M, K, dtype=BF16, device="cuda")
    x[-2:] = torch.randn(2, K, device="cuda", generator=g).to(BF16)
    y = torch.empty(M, N, dtype=BF16, device="cuda")
    uep.ultraep_expert_matmul_bf16(x, M, w, 1, N * K, N, K, trans, dev(np.array([0, M])), None, 1, 0, None, y, st)
    v = (w.view(K, N) if trans else w.view(N, K).t()).double().contiguous()
    want, mag = x[-2:].double() @ v, x[-2:].double().abs() @ v.abs()
    assert ((y[-2:].double() - want).abs() <= 2 * K * p64.U32 * mag + p64.U16 * want.abs() * 1.01).all()
    assert not y[:-2].any()


# ------------------------------------------------------------ weights' gradient

def check_weight_grad(sizes, N, K, f32, of=None, n_w=None, start=0, tail=0, gap=0, accumulate=False, ws=True, seed=0,
                      spoil=False):
    rng = np.random.default_rng(seed)
    off, M = layout(sizes, start, tail)
    n_w = n_w or len(sizes)
    dy, x = normal(rng, M, N), normal(rng, M, K)
    if spoil:
        for t in (dy, x):
            t[:off[0]] = t[off[-1]:] = np.nan
    dw = torch.full((n_w, N * K + gap), 7.0, dtype=F32 if f32 else BF16, device="cuda")
    old = np.zeros((n_w, N * K))
    if accumulate:
        dw[:, :N * K] = dev(normal(rng, n_w, N * K) * 3)
        old = dw[:, :N * K].double().cpu().numpy()  # as its type holds it
    ws = torch.empty(uep.ultraep_expert_weight_grad_ws_bytes(M, N, K, n_w), dtype=U8, device="cuda").fill_(255) if ws else None
    st = status()
    uep.ultraep_expert_weight_grad(dev16(dy), dev16(x), M, N, K, dev(off),
                                   None if of is None else dev(np.array(of, np.int32)), len(sizes), n_w, N * K + gap,
                                   accumulate, dw, ws, st)
    assert int(st.item()) == 0
    inside = slice(off[0], off[-1])
    want, err = pe.weight_grad(dy[inside].astype(np.float64), x[inside].astype(np.float64), off - off[0], of, n_w)
    want = want + old.reshape(want.shape)
    got = dw.double().cpu().numpy()
    assert (got[:, N * K:] == 7).all()
    got = got[:, :N * K].reshape(n_w, N, K)
    assert np.isfinite(got).all()
    # (the sum with what was there is one more rounding to fp32)
    same_where_defined(got, want, pe.rounded(want, err + p64.U32 * (np.abs(want) + err), f32))


@pytest.mark.parametrize("sizes,N,K", [
    ([1], 8, 8), ([0, 3, 0], 24, 40), ([65, 0, 63, 1], 72, 136), ([130, 7], 264, 72), ([257, 64], 144, 520),
    ([900], 264, 520), ([4000], 64, 64), ([3, 2500, 31], 128, 192), ([17] * 40, 136, 264), ([200, 100], 1032, 520)])
@pytest.mark.parametrize("f32", [True, False])
def test_weight_grad(sizes, N, K, f32):
    check_weight_grad(sizes, N, K, f32)


@pytest.mark.parametrize("sizes,N,K", [([300, 77], 2056, 2056), ([70, 0, 130, 1, 64, 9], 2056, 2056), ([33], 4104, 4104),
                                           ([300, 0, 513, 77], 2040, 2032), ([1, 65, 129, 64, 63], 2048, 2048)])
@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("accumulate", [True, False])
def test_weight_grad_of_large_weights(sizes, N, K, f32, accumulate):
    check_weight_grad(sizes, N, K, f32, accumulate=accumulate, gap=16)


def test_weight_grad_of_parts_over_many_blocks():
    """Few small weights, their rows in parts that begin and end inside blocks."""
    rng = np.random.default_rng(3)
    sizes = rng.integers(0, 200, 300)
    of = rng.integers(0, 3, 300)
    check_weight_grad(sizes.tolist(), 72, 136, True, of=of.tolist(), n_w=3)
    check_weight_grad(sizes.tolist(), 72, 136, True, of=of.tolist(), n_w=3, ws=False)


@pytest.mark.parametrize("accumulate", [True, False])
@pytest.mark.parametrize("sizes,of,n_w,N,K", [
    ([3000, 5, 0, 40, 9000], [0, 1, 2, 3, 4], 5, 200, 72), ([3000, 5, 0, 40, 9000, 64], [3, 1, 0, 3, 1, 0], 4, 136, 264),
    ([12000, 1, 0, 4400, 100], [0, 1, 2, 3, 4], 5, 2568, 264), ([2, 6000, 1], [0, 1, 2], 3, 8, 8)])
def test_weight_grad_of_parts_by_their_rows(sizes, of, n_w, N, K, accumulate):
    """Weights with nearly all rows, with a few and with none, in parts by their rows."""
    check_weight_grad(sizes, N, K, accumulate, of=of, n_w=n_w, gap=8, start=3, tail=70, spoil=True, accumulate=accumulate)


def test_weight_grad_of_parts_of_many_weights():
    rng = np.random.default_rng(9)
    sizes = rng.integers(0, 900, 600)
    sizes[7] = 20000
    of = rng.integers(0, 256, 600)
    of[sizes == 0] = -1
    check_weight_grad(sizes.tolist(), 64, 64, True, of=of.tolist(), n_w=256)


@pytest.mark.parametrize("f32", [True, False])
@pytest.mark.parametrize("ws", [True, False])
def test_weight_grad_accumulates(f32, ws):
    check_weight_grad([100, 0, 37], 136, 200, f32, accumulate=True, gap=40, ws=ws)
    check_weight_grad([2000, 0, 3000], 64, 72, f32, accumulate=True, gap=40, ws=ws)


@pytest.mark.parametrize("accumulate", [True, False])
def test_weight_grad_of_shared_weights_and_spare_rows(accumulate):
    """Weights 1 and 3 have no rows; two blocks each of 0 and 2; NaN outside the blocks."""
    check_weight_grad([40, 0, 33, 90, 70], 72, 96, True, of=[2, 9, 0, 2, 0], n_w=4, start=5, tail=9, spoil=True,
                      accumulate=accumulate)
    check_weight_grad([1500, 0, 33, 2000, 700], 72, 96, True, of=[2, 9, 0, 2, 0], n_w=4, start=5, tail=9, spoil=True,
                      accumulate=accumulate)


def test_weight_grad_of_many_blocks():
    rng = np.random.default_rng(2)
    sizes = rng.integers(0, 5, 2048)
    sizes[[3, 700, 2047]] = [150, 0, 65]
    of = rng.integers(0, 6, 2048)
    of[sizes == 0] = -7
    check_weight_grad(sizes.tolist(), 40, 72, True, of=of.tolist(), n_w=6)


def test_weight_grad_without_rows():
    dw, st = torch.full((2, 16, 24), 7.0, device="cuda"), status()
    off = torch.zeros(3, dtype=I64, device="cuda")
    uep.ultraep_expert_weight_grad(None, None, 0, 16, 24, off, None, 2, 2, 16 * 24, True, dw, None, st)
    assert (dw == 7).all()
    uep.ultraep_expert_weight_grad(None, None, 0, 16, 24, off, None, 2, 2, 16 * 24, False, dw, None, st)
    assert int(st.item()) == 0 and (dw == 0).all()


def test_weight_grad_of_other_numbers():
    """An infinity and a NaN reach their row and column of their weight alone; zeros
    beside them are multiplied by them too."""
    rng = np.random.default_rng(9)
    M, N, K = 90, 24, 40
    dy, x = normal(rng, M, N), normal(rng, M, K)
    dy[3, 5], x[50, 7], x[60, 9] = np.nan, np.inf, np.nan
    dy[50, 2] = 0.0
    off = np.array([0, 40, 90])
    with np.errstate(invalid="ignore"):
        want, _ = pe.weight_grad(dy.astype(np.float64), x.astype(np.float64), off, None, 2)
    dw = torch.empty(2, N, K, device="cuda")
    uep.ultraep_expert_weight_grad(dev16(dy), dev16(x), M, N, K, dev(off), None, 2, 2, N * K, False, dw, None, status())
    got = dw.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[np.isinf(want)], want[np.isinf(want)])


def test_weight_grad_of_a_side_with_itself_is_symmetric():
    rng = np.random.default_rng(10)
    x = dev16(normal(rng, 300, 72))
    dw = torch.empty(1, 72, 72, device="cuda")
    uep.ultraep_expert_weight_grad(x, x, 300, 72, 72, dev(np.array([0, 300])), None, 1, 1, 72 * 72, False, dw, None, status())
    assert torch.equal(dw[0], dw[0].t())


def test_weight_grad_offsets_past_32_bits():
    """Rows of over 4 GiB on either side, gradients of over 4 GiB."""
    M, N, K = 600_000, 4096, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    big, small = torch.zeros(M, N, dtype=BF16, device="cuda"), torch.randn(M, K, device="cuda", generator=g).to(BF16)
    big[-3:] = torch.randn(3, N, device="cuda", generator=g).to(BF16)
    off = dev(np.array([0, M - 2, M]))
    dw = torch.empty(2, N, K, device="cuda")
    for _ in range(2):
        uep.ultraep_expert_weight_grad(big, small, M, N, K, off, None, 2, 2, N * K, False, dw, None, status())
    a, b = big[-3:].double(), small[-3:].double()
    for i, r in ((0, slice(0, 1)), (1, slice(1, 3))):
        want, mag = a[r].t() @ b[r], a[r].abs().t() @ b[r].abs()
        assert ((dw[i] - want).abs() <= 8 * p64.U32 * mag + 1e-37).all()
    dw2 = torch.empty(2, K, N, device="cuda")
    uep.ultraep_expert_weight_grad(small, big, M, K, N, off, None, 2, 2, N * K, False, dw2, None, status())
    want, mag = b[1:].t() @ a[1:], b[1:].abs().t() @ a[1:].abs()
    assert ((dw2[1] - want).abs() <= 8 * p64.U32 * mag + 1e-37).all()
    del big, small
    N, K = 16384, 32768
    y, x = torch.randn(3, N, device="cuda", generator=g).to(BF16), torch.randn(3, K, device="cuda", generator=g).to(BF16)
    dw = torch.empty(5, N * K, dtype=BF16, device="cuda")
    uep.ultraep_expert_weight_grad(y, x, 3, N, K, dev(np.array([0, 3])), dev(np.array([4], np.int32)), 1, 5, N * K, False,
                                   dw, None, status())
    assert not dw[:4].any()
    got = dw[4].view(N, K)
    for lo in range(0, N, 2048):
        want = y[:, lo:lo + 2048].double().t() @ x.double()
        mag = y[:, lo:lo + 2048].double().abs().t() @ x.double().abs()
        assert ((got[lo:lo + 2048].double() - want).abs() <= 8 * p64.U32 * mag + 1.01 * p64.U16 * want.abs() + 1e-37).all()


# ---------------------------------------------------------- block quantisation

@pytest.mark.parametrize("rows,K,ld,ldq", [
    (1, 8, 8, 16), (1, 16, 16, 16), (3, 24, 40, 32), (65, 520, 520, 528), (257, 2888, 2896, 2896), (5, 128, 128, 128),
    (7, 136, 136, 400), (40, 7168, 7168, 7168), (9, 12288, 12296, 12304), (3, 65536, 65536, 65536), (1000, 64, 72, 128),
    (17000, 520, 528, 528), (11000, 1160, 1160, 1168), (6600, 2312, 2312, 2560)])
@pytest.mark.parametrize("bf16", [True, False])
def test_quant_blocks(rows, K, ld, ldq, bf16):
    rng = np.random.default_rng(rows * K)
    x = (rng.standard_normal((rows, ld)) * np.exp(4 * rng.standard_normal((rows, 1)))).astype(np.float32)
    x[:, K:] = np.nan  # what lies between rows is not looked at
    if rows > 4:
        x[1, :K] = 0
        x[2, :K] *= np.float32(1e-38)
        x[3, :K] *= np.float32(1e33)
    if bf16:
        x = p64.bf16(x)
    n = uep.scale_pitch(K)
    q = torch.full((rows * ldq + 64,), 55, dtype=U8, device="cuda")
    s = torch.full((rows * n + 8,), 5, dtype=U8, device="cuda")
    uep.ultraep_quant_blocks(dev16(x) if bf16 else dev(x), rows, K, ld, q, ldq, s)
    rq, rs = pe.quant_blocks(x[:, :K], ldq)
    assert np.array_equal(s[:rows * n].cpu().numpy().reshape(rows, n), rs)
    assert np.array_equal(q[:rows * ldq].cpu().numpy().reshape(rows, ldq), rq)
    assert (q[rows * ldq:] == 55).all() and (s[rows * n:] == 5).all()


@pytest.mark.parametrize("bf16", [True, False])
def test_quant_blocks_of_other_numbers(bf16):
    """Infinities, NaN, the type's largest and smallest values, zeros of both signs, exact
    halves (to even), and maxima on either side of 448 times a power of two."""
    x = np.zeros((20, 136), np.float32)
    x[0, 3] = np.inf
    x[1, 131] = -np.inf
    x[2, 0] = np.nan
    x[3] = -0.0
    x[4] = np.linspace(-1, 1, 136) * 3.3e38
    x[5, :6] = [448, 17, 19, 21, -17, -19]
    x[6, :3] = [448, 2.0 ** -10, 3 * 2.0 ** -10]
    x[7, :2] = [448 * 1.01, 1]
    x[8, :2] = [447, 1]
    x[9, 0], x[10, 0] = 2.0 ** -126, 1e-45
    x[11, :2] = [448 * 2.0 ** -127, 448 * 2.0 ** -130]
    x[12, 130] = 896
    x[13, 130] = 896.0001
    x[14] = 240
    x[15] = np.finfo(np.float32).max
    if bf16:
        x = p64.bf16(np.minimum(x, 3.3e38)) if np.isfinite(x).all() else p64.bf16(x)
    q, s = torch.empty(20, 144, dtype=U8, device="cuda"), torch.empty(20, 4, dtype=U8, device="cuda")
    uep.ultraep_quant_blocks(dev16(x) if bf16 else dev(x), 20, 136, 136, q, 144, s)
    rq, rs = pe.quant_blocks(x, 144)
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), rq)
    assert rs[0, 0] == 255 and rs[1].tolist() == [0, 255, 0, 0] and rs[5, 0] == 127 and rs[8, 0] == 127


def test_quant_blocks_offsets_past_32_bits():
    rows, K = 300_001, 8192
    x = torch.zeros(rows, K, dtype=BF16, device="cuda")
    x[-3:] = torch.randn(3, K, device="cuda").to(BF16)
    q, s = torch.empty(rows, K, dtype=U8, device="cuda"), torch.empty(rows, 64, dtype=U8, device="cuda")
    uep.ultraep_quant_blocks(x, rows, K, K, q, K, s)
    rq, rs = pe.quant_blocks(x[-3:].float().cpu().numpy(), K)
    assert np.array_equal(q[-3:].cpu().numpy(), rq) and np.array_equal(s[-3:].cpu().numpy(), rs)
    assert not q[:-3].any() and not s[:-3].any()


# -------------------------------------------------------------- 8-bit products

def e4m3_rows(rng, rows, K, spread=2.0):
    x = (rng.standard_normal((rows, K)) * np.exp(spread * rng.standard_normal((rows, K // 16)).repeat(16, axis=1)))
    return pe.quant_blocks(x.astype(np.float32), K)


def fp8_product(sizes, N, K, act, f32, of=None, n_w=None, start=0, tail=0, seed=0, spoil=None, whole=False):
    rng = np.random.default_rng(seed)
    off, M = layout(sizes, start, tail)
    n_w = n_w or len(sizes)
    (xq, xs), (wq, ws) = e4m3_rows(rng, M, K), e4m3_rows(rng, n_w * N, K)
    if whole:  # small integers: every product and sum is exact
        digits = pe.e4m3_bits(np.arange(-3.0, 4.0))
        xq, wq = rng.choice(digits, xq.shape), rng.choice(digits, wq.shape)
        xs, ws = np.where(xs > 0, 127, 0).astype(np.uint8), np.where(ws > 0, 126, 0).astype(np.uint8)
    wq, ws = wq.reshape(n_w, N, K), ws.reshape(n_w, N, -1)
    if spoil:
        spoil(xq, xs, wq, ws)
    y = torch.full((M, N // 2 if act == "swiglu" else N), 3.0, dtype=F32 if f32 else BF16, device="cuda")
    st = status()
    uep.ultraep_expert_matmul_fp8(dev(xq), dev(xs), M, dev(wq), dev(ws), n_w, N, K, dev(off),
                                  None if of is None else dev(np.array(of, np.int32)), len(sizes), ACTS[act], y, st)
    assert int(st.item()) == 0
    want, err, _, _ = pe.product(pe.dequantised(xq, xs), pe.dequantised(wq, ws), off, of, act, cut=not f32, taken_to_bf16=f32)
    if whole:
        err = np.zeros_like(err)
    got = y.double().cpu().numpy()
    inside = np.zeros(M, bool)
    inside[off[0]:off[-1]] = True
    assert (got[~inside] == 3).all()
    return got[inside], want[inside], pe.rounded(want, err, f32)[inside]


SHAPES8 = [
    ([1], 16, 16), ([1], 64, 4096), ([0, 3, 0], 48, 48), ([65, 0, 63, 1], 96, 144), ([130, 7], 272, 272),
    ([5, 64, 128, 200], 144, 528), ([257], 528, 128), ([300, 300], 320, 400), ([16] * 4, 1040, 2064), ([40], 64, 3600),
    ([200], 2064, 144)
] + [(s, n // 16 * 16, k // 16 * 16) for s, n, k in TILES]


@pytest.mark.parametrize("sizes,N,K", SHAPES8)
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_fp8_products(sizes, N, K, act):
    got, want, err = fp8_product(sizes, N, K, act, False, **shared(sizes))
    assert np.isfinite(got).all()
    same_where_defined(got, want, err)


@pytest.mark.parametrize("sizes,N,K", SHAPES8)
@pytest.mark.parametrize("f32", [False, True])
def test_fp8_products_of_small_integers_are_exact(sizes, N, K, f32):
    """Products of at most 9 are summed without a rounding, so every element that a wrong
    place would bring is seen; a bf16 result is the exact one's rounding."""
    got, want, _ = fp8_product(sizes, N, K, "none", f32, whole=True, **shared(sizes))
    if not f32:
        want = p64.bf16(want.astype(np.float32)).astype(np.float64)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("sizes,N,K", [(s, n // 16 * 16, k // 16 * 16) for s, n, k in TILES])
def test_fp8_products_fp32_results_over_the_tile_shapes(sizes, N, K):
    got, want, err = fp8_product(sizes, N, K, "swiglu", True, **shared(sizes))
    assert np.isfinite(got).all()
    same_where_defined(got, want, err)


@pytest.mark.parametrize("sizes,N,K", [(s, n // 16 * 16, k // 16 * 16) for s, n, k in MANY])
@pytest.mark.parametrize("act,f32", [("none", False), ("swiglu", False), ("none", True)])
def test_fp8_products_of_many_tiles(sizes, N, K, act, f32):
    got, want, err = fp8_product(sizes, N, K, act, f32, **shared(sizes))
    assert np.isfinite(got).all()
    same_where_defined(got, want, err)


@pytest.mark.parametrize("sizes,N,K", [([70, 3], 80, 48), ([1], 32, 528), ([300, 41], 336, 144)])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_fp8_products_fp32_results(sizes, N, K, act):
    got, want, err = fp8_product(sizes, N, K, act, True, start=3, tail=4)
    assert np.isfinite(got).all()
    same_where_defined(got, want, err)


def test_fp8_products_of_shared_weights_and_many_blocks():
    got, want, err = fp8_product([40, 0, 33, 90], 64, 96, "none", False, of=[2, 7, 0, 2], n_w=3, start=5, tail=9)
    same_where_defined(got, want, err)
    rng = np.random.default_rng(1)
    sizes = rng.integers(0, 4, 2048)
    of = rng.integers(0, 5, 2048)
    of[sizes == 0] = -7
    got, want, err = fp8_product(sizes.tolist(), 32, 48, "none", False, of=of.tolist(), n_w=5)
    same_where_defined(got, want, err)


@pytest.mark.parametrize("K", [16, 112, 144, 272])
def test_fp8_products_of_other_numbers(K):
    """NaN values and scales stay in their row and channel; what lies outside the blocks
    and in other weights is not looked at; scales of 2^-127 and 2^100."""
    def spoil(xq, xs, wq, ws):
        xq[:2] = xq[-3:] = 0x7F
        wq[0] = wq[2] = 0x7F
        xq[5, K - 1], xs[6, 0] = 0xFF, 255
        wq[1, 9, 3], ws[1, 10, (K - 1) // 128] = 0x7F, 255
        xs[7] = 0
        ws[1, 11] = 227
    got, want, err = fp8_product([21], 40, K, "none", True, of=[1], n_w=3, start=2, tail=3, spoil=spoil)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any() and not np.isnan(want).all()
    same_where_defined(got, want, err)


@pytest.mark.parametrize("M", [5, 300])
@pytest.mark.parametrize("bytes_", [(0, 254), (254, 0), (1, 253), (254, 127), (127, 0)])
@pytest.mark.parametrize("f32", [False, True])
def test_fp8_products_of_the_least_and_largest_scales(M, bytes_, f32):
    """0, 1 and -1 (2 and -2 under scale 2^-127, so that bf16 holds them too): sums of 144 are exact."""
    rng = np.random.default_rng(6)
    N, K = 80, 144
    def side(rows, byte):
        digits = pe.e4m3_bits(np.array([-1.0, 0.0, 1.0]) * (2 if byte == 0 else 1))
        s = np.zeros((rows, uep.scale_pitch(K)), np.uint8)
        s[:, :2] = byte
        return rng.choice(digits, (rows, K)), s
    (xq, xs), (wq, ws) = side(M, bytes_[0]), side(N, bytes_[1])
    if bytes_ == (254, 127):  # sums of several would be infinite
        xq[:, 1:] = 0
    y, st = torch.empty(M, N, dtype=F32 if f32 else BF16, device="cuda"), status()
    uep.ultraep_expert_matmul_fp8(dev(xq), dev(xs), M, dev(wq), dev(ws), 1, N, K, dev(np.array([0, M])), None, 1,
                                  uep.ULTRAEP_NO_ACT, y, st)
    want = pe.dequantised(xq, xs) @ pe.dequantised(wq, ws).T
    if not f32:
        want = p64.bf16(want.astype(np.float32)).astype(np.float64)
    assert want.any() and np.array_equal(y.double().cpu().numpy(), want)


def test_fp8_products_offsets_past_32_bits():
    n_w, N, K = 5, 32768, 32768
    g = torch.Generator(device="cuda").manual_seed(2)
    w = torch.zeros(n_w, N, K, dtype=U8, device="cuda")
    ws = torch.full((n_w, N, 256), 127, dtype=U8, device="cuda")
    w[4] = torch.randint(0x20, 0x40, (N, K), dtype=U8, device="cuda", generator=g)
    x = torch.randint(0x20, 0x40, (3, K), dtype=U8, device="cuda", generator=g)
    xs = torch.randint(120, 130, (3, 256), dtype=U8, device="cuda", generator=g)
    y, st = torch.empty(3, N, device="cuda"), status()
    uep.ultraep_expert_matmul_fp8(x, xs, 3, w, ws, n_w, N, K, dev(np.array([0, 1, 3])), dev(np.array([4, 4], np.int32)), 2, 0,
                                  y, st)
    xd = torch.from_numpy(pe.dequantised(x.cpu().numpy(), xs.cpu().numpy())).cuda()
    want = torch.zeros(3, N, dtype=torch.float64, device="cuda")
    for k in range(0, K, 4096):
        want += xd[:, k:k + 4096] @ w[4][:, k:k + 4096].contiguous().view(torch.float8_e4m3fn).to(F32).double().t().contiguous()
    assert int(st.item()) == 0 and ((y - want).abs() <= 2 * K * p64.U32 * want).all()  # (all terms are positive)
