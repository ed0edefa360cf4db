"""The experts' operators together, as a training step and a serving step use them: both
products of a gated expert with what the first keeps, their gradients back to the rows and
the weights, which lie in one blob an expert; quantisation, product, quantisation, product
in 8-bit floating point.  Every stage is compared with the plain 64-bit implementation of
it on what the stage before left, within the bounds that plain_experts derives; the ends
with torch's gradients in 64 bits.  Needs an MI355X."""
import numpy as np
import pytest
import torch

import plain64 as p64
import plain_experts as pe
from test_gpu_expert_products import dev, dev16, layout, normal, same_where_defined, status

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

F32, BF16, U8 = torch.float32, torch.bfloat16, torch.uint8


class Experts:
    """n_w experts, up [2F][H] (gates first) and down [H][F] one after the other in a blob
    of W elements; the buffers of a step over blocks of rows."""

    def __init__(self, sizes, of, n_w, H, F, start=0, tail=0, seed=0):
        rng = np.random.default_rng(seed)
        self.H, self.F, self.n_w, self.of = H, F, n_w, of
        self.off, self.M = layout(sizes, start, tail)
        self.inside = slice(int(self.off[0]), int(self.off[-1]))
        self.W = 3 * F * H + 24  # and something else behind them
        self.up = normal(rng, n_w, 2 * F, H) * np.float32(2.0 ** -3)
        self.down = normal(rng, n_w, H, F) * np.float32(2.0 ** -3)
        blob = np.full((n_w, self.W), np.nan, np.float32)
        blob[:, :2 * F * H] = self.up.reshape(n_w, -1)
        blob[:, 2 * F * H:3 * F * H] = self.down.reshape(n_w, -1)
        self.blob = dev16(blob)
        self.blob_down = self.blob.reshape(-1)[2 * F * H:]
        self.x, self.dy = dev16(self.rows(rng)), dev16(self.rows(rng))
        self.blocks = dev(self.off), dev(np.array(of, np.int32)), len(sizes)
        M = self.M
        self.pre, self.h, self.y, self.dpre, self.dx = (
            torch.full((M, n), 7.0, dtype=BF16, device="cuda") for n in (2 * F, F, H, 2 * F, H))
        self.grad = torch.full((n_w, self.W), 7.0, dtype=F32, device="cuda")
        self.ws = [torch.empty(uep.ultraep_expert_weight_grad_ws_bytes(M, *s, n_w), dtype=U8, device="cuda")
                   for s in ((2 * F, H), (H, F))]
        self.status = status()

    def rows(self, rng):
        r = np.full((self.M, self.H), np.nan, np.float32)
        r[self.inside] = normal(rng, self.inside.stop - self.inside.start, self.H)
        return r

    def product(self, x, w, N, K, trans, act, pre, y):
        uep.ultraep_expert_matmul_bf16(x, self.M, w, self.n_w, self.W, N, K, trans, *self.blocks, act, pre, y, self.status)

    def weight_grad(self, dy, x, N, K, ws, dw, accumulate):
        uep.ultraep_expert_weight_grad(dy, x, self.M, N, K, *self.blocks, self.n_w, self.W, accumulate, dw, ws, self.status)

    def step(self, accumulate=False):
        H, F = self.H, self.F
        grad_down = self.grad.view(-1)[2 * F * H:]
        self.product(self.x, self.blob, 2 * F, H, False, uep.ULTRAEP_SWIGLU, self.pre, self.h)
        self.product(self.h, self.blob_down, H, F, False, uep.ULTRAEP_NO_ACT, None, self.y)
        self.weight_grad(self.dy, self.h, H, F, self.ws[1], grad_down, accumulate)
        self.product(self.dy, self.blob_down, F, H, True, uep.ULTRAEP_SWIGLU_GRAD, self.pre, self.dpre)
        self.weight_grad(self.dpre, self.x, 2 * F, H, self.ws[0], self.grad, accumulate)
        self.product(self.dpre, self.blob, H, 2 * F, True, uep.ULTRAEP_NO_ACT, None, self.dx)

    def results(self):
        return [t.clone() for t in (self.pre, self.h, self.y, self.dpre, self.dx, self.grad)]


def f64(t):
    return t.view(BF16).double().cpu().numpy() if t.element_size() == 2 else t.double().cpu().numpy()


CASES = [  # blocks over their weights; a weight without rows; few small weights, whose rows are summed in parts
    dict(sizes=[0, 3, 300, 1, 64], of=[4, 2, 0, 2, 1], n_w=4, H=72, F=40, start=3, tail=5),
    dict(sizes=[1500, 0, 33, 2000, 700], of=[1, -1, 0, 0, 1], n_w=2, H=64, F=48, start=0, tail=9),
    dict(sizes=[1], of=[0], n_w=1, H=128, F=16),
    dict(sizes=[130, 257, 129, 511], of=[0, 1, 2, 3], n_w=4, H=520, F=264)]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_a_training_step(case):
    e = Experts(**CASES[case])
    H, F, W, ins, off, of = e.H, e.F, e.W, e.inside, e.off, e.of
    e.step()
    assert int(e.status.item()) == 0
    for t in e.results()[:5]:  # rows outside the blocks are left alone
        outside = torch.cat([t[:ins.start], t[ins.stop:]])
        assert (outside == 7).all()
    assert (e.grad[:, 3 * F * H:] == 7).all()
    x, dy, pre, h, dpre = (f64(t) for t in (e.x, e.dy, e.pre, e.h, e.dpre))
    up, down = e.up.astype(np.float64), e.down.astype(np.float64)

    def near(got, want, err, f32=False):
        same_where_defined(f64(got)[ins], want[ins], pe.rounded(want, err, f32)[ins])

    want, err, v, dv = pe.product(x, up, off, of, "swiglu")
    near(e.h, want, err)
    near(e.pre, v, dv)
    near(e.y, *pe.product(h, down, off, of, "none")[:2])
    near(e.dpre, *pe.product(dy, down, off, of, "swiglu_grad", True, pre)[:2])
    near(e.dx, *pe.product(dpre, up, off, of, "none", True)[:2])
    got = f64(e.grad)
    for a, b, at, shape in ((dy, h, 2 * F * H, (H, F)), (dpre, x, 0, (2 * F, H))):
        want, err = pe.weight_grad(a[ins], b[ins], off - off[0], of, e.n_w)
        same_where_defined(got[:, at:at + shape[0] * shape[1]].reshape(want.shape), want, pe.rounded(want, err, True))
    # A second microbatch of the same rows on top: twice the gradient, which is exact in fp32
    # but for the sums' last rounding.
    first = e.grad.clone()
    e.step(accumulate=True)
    rel = (e.grad[:, :3 * F * H] - 2 * first[:, :3 * F * H]).abs() <= 2.0 ** -23 * first[:, :3 * F * H].abs()
    assert rel.all() and (e.grad[:, 3 * F * H:] == 7).all()


@pytest.mark.parametrize("case", range(len(CASES)))
def test_gradients_against_torch_in_64_bits(case):
    """The ends of the chain: y through h, dx and the weights' gradients through h, pre and
    dpre, each rounded once to bf16 (half a step, 2^-8) on the way and the result once more:
    at most five roundings, below 0.02 of a norm."""
    e = Experts(**CASES[case])
    e.step()
    H, F, ins = e.H, e.F, e.inside
    x = torch.from_numpy(f64(e.x)).requires_grad_()
    up, down = (torch.from_numpy(t.astype(np.float64)).requires_grad_() for t in (e.up, e.down))
    y = []
    for g, w in enumerate(e.of):
        lo, hi = e.off[g], e.off[g + 1]
        if hi > lo:
            a, u = (x[lo:hi] @ up[w].t()).chunk(2, 1)
            y.append((torch.nn.functional.silu(a) * u) @ down[w].t())
    y = torch.cat(y)
    y.backward(torch.from_numpy(f64(e.dy))[ins])
    grad = e.grad.double().cpu()
    for got, want in ((e.y.double().cpu()[ins], y.detach()), (e.dx.double().cpu()[ins], x.grad[ins]),
                      (grad[:, :2 * F * H], up.grad.flatten(1)), (grad[:, 2 * F * H:3 * F * H], down.grad.flatten(1))):
        assert float((got - want).norm()) <= 0.02 * float(want.norm())


@pytest.mark.parametrize("case", [0, 1, 3])
def test_a_captured_training_step(case):
    """The step as a graph, replayed over changing rows with eager steps between."""
    e, other = Experts(**CASES[case]), Experts(**CASES[case], seed=1)
    wants = []
    for src in (e.x.clone(), other.x):
        e.x.copy_(src)
        e.step()
        wants.append((src, e.results()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e.step()
    for src, want in wants * 2:
        e.x.copy_(src)
        e.grad[:, :3 * e.F * e.H] = 0
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(e.results(), want))
        e.step()
        assert all(torch.equal(a, b) for a, b in zip(e.results(), want))
    assert int(e.status.item()) == 0


@pytest.mark.parametrize("sizes,of,n_w,H,F", [([0, 3, 200, 1, 64], [3, 2, 0, 2, 1], 4, 144, 80), ([1], [0], 1, 528, 272),
                                              ([700, 300], [1, 0], 2, 256, 400)])
def test_a_serving_step_in_8_bits(sizes, of, n_w, H, F):
    rng = np.random.default_rng(2)
    off, M = layout(sizes, 0, 2)
    n = int(off[-1])
    blocks, st = (dev(off), dev(np.array(of, np.int32)), len(sizes)), status()

    def quantised(t, rows, K):
        t = t.view(BF16)
        q = torch.empty(rows, K, dtype=U8, device="cuda")
        s = torch.empty(rows, uep.scale_pitch(K), dtype=U8, device="cuda")
        uep.ultraep_quant_blocks(t, rows, K, K, q, K, s)
        return q, s, pe.dequantised(q.cpu().numpy(), s.cpu().numpy())
    x = normal(rng, M, H)
    up, down = normal(rng, n_w, 2 * F, H) * np.float32(2.0 ** -3), normal(rng, n_w, H, F) * np.float32(2.0 ** -3)
    uq, us, u64 = quantised(dev16(up), n_w * 2 * F, H)
    dq, ds, d64 = quantised(dev16(down), n_w * H, F)
    xq, xs, x64 = quantised(dev16(x), M, H)
    h, y = torch.zeros(M, F, dtype=BF16, device="cuda"), torch.zeros(M, H, dtype=BF16, device="cuda")
    uep.ultraep_expert_matmul_fp8(xq, xs, M, uq, us, n_w, 2 * F, H, *blocks, uep.ULTRAEP_SWIGLU, h, st)
    hq, hs, h64 = quantised(h, M, F)
    uep.ultraep_expert_matmul_fp8(hq, hs, M, dq, ds, n_w, H, F, *blocks, uep.ULTRAEP_NO_ACT, y, st)
    assert int(st.item()) == 0
    want, err, _, _ = pe.product(x64, u64.reshape(n_w, 2 * F, H), off, of, "swiglu", cut=True)
    same_where_defined(f64(h)[:n], want[:n], pe.rounded(want, err, False)[:n])
    want, err, _, _ = pe.product(h64, d64.reshape(n_w, H, F), off, of, "none", cut=True)
    same_where_defined(f64(y)[:n], want[:n], pe.rounded(want, err, False)[:n])
    # The blocks of rows that end behind the list's last: zeros as they were.
    assert not h[n:].any() and not y[n:].any()
    # Against the layer of unrounded values: a rounding to e4m3 is off by 2^-4 at most and by 0.024
    # of the root mean square (step / sqrt(12) over a binade); x and the up weights reach h through
    # both factors (0.024 * sqrt(2) each, 0.05 in all), h and the down weights add 0.024 each: 0.06.
    plain = np.zeros((M, H))
    for g, w in enumerate(of):
        rows = slice(off[g], off[g + 1])
        plain[rows] = pe.swiglu(x[rows].astype(np.float64) @ up[w].T.astype(np.float64)) @ down[w].T.astype(np.float64) \
            if off[g + 1] > off[g] else 0
    assert np.linalg.norm(f64(y)[:n] - plain[:n]) < 0.1 * np.linalg.norm(plain[:n])
