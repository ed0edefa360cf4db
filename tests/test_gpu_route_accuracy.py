"""The router's numbers where fp32 loses them first: logits so high that 1 minus
a sigmoid score cancels.  Against 64-bit formulas that take 1 - s as sigmoid(-z).
Needs an MI355X.

Tolerances, in units of u = 2^-24: a score or its complement is under 100 u off
(|z| u by exp's argument, |z| <= 32 here, 2 ulp by exp, the sums over E, three
products and quotients), and an element of the gradient carries two of them on
each of the terms whose magnitudes `mag` sums; bf16 adds half an ulp."""
import numpy as np
import pytest
import torch

import plain64 as p64

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

SCORE_U = 100 * p64.U32


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def sigmoid_grad(z, ids, scale, renorm, dg, w):
    """dlogits [T][E] of a sigmoid router and the sums of its terms' magnitudes, in
    64 bits; every id is an expert."""
    s, rest = p64.sigmoid(z), p64.sigmoid(-z)
    p = s / s.sum(1, keepdims=True)
    dz = p * rest * (w - (w * p).sum(1, keepdims=True))
    mag = p * rest * (np.abs(w) + (np.abs(w) * p).sum(1, keepdims=True))
    si, ri = np.take_along_axis(s, ids, 1), np.take_along_axis(rest, ids, 1)
    dg = dg * scale
    if renorm:
        q = si / si.sum(1, keepdims=True)
        d = q * ri * (dg - (q * dg).sum(1, keepdims=True))
        m = q * ri * (np.abs(dg) + (q * np.abs(dg)).sum(1, keepdims=True))
    else:
        d, m = si * ri * dg, si * ri * np.abs(dg)
    for j in range(ids.shape[1]):
        t = np.arange(len(z))
        dz[t, ids[:, j]] += d[:, j]
        mag[t, ids[:, j]] += m[:, j]
    return dz, mag


def test_the_formula_against_differences():
    rng = np.random.default_rng(4)
    E, k, h = 12, 3, 1e-4
    for renorm in (True, False):
        r = dict(E=E, k=k, score="sigmoid", renorm=renorm, n_group=0, top_group=0, scale=2.5, seq_len=0)
        z = rng.uniform(-3, 9, (4, E))
        ids = np.argsort(-z, axis=1)[:, :k]
        dg, w = rng.standard_normal((4, k)), rng.standard_normal((4, E))
        got, _ = sigmoid_grad(z, ids, 2.5, renorm, dg, w)
        for t in range(4):
            for e in range(E):
                hi, lo = z[t].copy(), z[t].copy()
                hi[e] += h
                lo[e] -= h
                d = (p64.objective(hi, ids[t], r, dg[t], w[t]) - p64.objective(lo, ids[t], r, dg[t], w[t])) / (2 * h)
                # h^2 / 6 of a third derivative of at most 10, and rounding, 1e-15 / h
                assert abs(d - got[t, e]) < 1e-7


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("parts", ["gates", "loss", "both"])
@pytest.mark.parametrize("E,k,T", [(256, 8, 40), (256, 8, 6200), (60, 4, 2100), (20, 4, 50), (512, 12, 33)])
def test_gradient_of_high_logits(E, k, T, parts, renorm, bf16):
    """A token's logits around 8 to 30, so that 1 - s is 3e-4 to 1e-13 of it; a part
    of them around 0."""
    rng = np.random.default_rng(E + T)
    z = (rng.uniform(8, 30, (T, 1)) + rng.uniform(-2, 2, (T, E))).astype(np.float32)
    z[rng.random((T, E)) < 0.2] -= np.float32(20)
    z = p64.bf16(z) if bf16 else z
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :k].astype(np.int32)
    dg = rng.standard_normal((T, k)).astype(np.float32)
    w = (10 * rng.standard_normal((1, E))).astype(np.float32)
    lg = dev(p64.bf16_bits(z).view(np.int16)) if bf16 else dev(z)
    out, st = torch.full_like(lg, 5), torch.zeros(1, dtype=torch.int32, device="cuda")
    uep.ultraep_route_grad(lg, T, E, uep.Router(E, k, uep.ULTRAEP_SIGMOID, renorm, scale=2.5), None, dev(ids),
                           dev(dg) if parts != "loss" else None, dev(w) if parts != "gates" else None, None, out, st)
    assert int(st.item()) == 0
    got = out.cpu().numpy()
    got = p64.from_bits(got.view(np.uint16)) if bf16 else got
    want, mag = sigmoid_grad(z.astype(np.float64), ids, 2.5, renorm, dg.astype(np.float64) * (parts != "loss"),
                             w.astype(np.float64) * (parts != "gates"))
    tol = 2 * SCORE_U * mag + 1e-37 + (1.01 * p64.U16 * np.abs(want) if bf16 else 0)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), float((np.abs(got - want) / mag.clip(1e-300)).max() / p64.U32))


def scores(z, score, renorm, k, st):
    """Gates and a token's own p by the kernel: every token a sequence."""
    T, E = z.shape
    r = uep.Router(E, k, uep.ULTRAEP_SIGMOID if score == "sigmoid" else uep.ULTRAEP_SOFTMAX, renorm, seq_len=1)
    i, f = torch.int32, torch.float32
    o = [torch.empty(s, dtype=d, device="cuda") for s, d in
         (((T, k), i), ((T, k), f), ((T, E), i), ((T, E), f), ((T,), i))]
    ws = torch.empty(uep.ultraep_route_ws_bytes(T, r), dtype=torch.uint8, device="cuda")
    uep.ultraep_route(dev(z), T, E, r, None, None, *o, ws, st)
    return o[0].cpu().numpy(), o[1].cpu().numpy(), o[3].cpu().numpy()


@pytest.mark.parametrize("E", [24, 256, 512])
def test_sigmoid_scores_of_low_and_high_logits(E):
    """Gates that are scores: exp within 2 ulp (4 u), 1 + exp (1 u and at most half of
    exp's), the reciprocal 1 ulp, a product; 10 u whatever the logit."""
    rng = np.random.default_rng(E)
    z = rng.uniform(-80, 20, (300, E)).astype(np.float32)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    k = min(E, 64)
    ids, gate, _ = scores(z, "sigmoid", False, k, st)
    want = p64.sigmoid(np.take_along_axis(z, ids, 1).astype(np.float64))
    assert int(st.item()) == 0 and (ids >= 0).all()
    assert (np.abs(gate - want) <= 10 * p64.U32 * want).all()
    low = np.where(rng.random((300, E)) < 0.5, z, z - np.float32(20)).clip(max=-2)  # down to -100, where exp is 0
    ids, gate, _ = scores(low, "sigmoid", False, k, st)
    want = p64.sigmoid(np.take_along_axis(low, ids, 1).astype(np.float64))
    assert (np.abs(gate - want) <= 10 * p64.U32 * want + 2.0 ** -126).all()


@pytest.mark.parametrize("E", [24, 256, 512])
def test_softmax_scores_far_below_the_largest(E):
    """One logit 30 to 80 above the others, differences exact: the sum is 1, a score exp
    (4 u), the reciprocal and a product (3 u); 8 u however small."""
    rng = np.random.default_rng(E)
    z = -rng.integers(30 * 16, 80 * 16, (300, E)).astype(np.float32) / 16
    z[np.arange(300), rng.integers(0, E, 300)] = 0
    z += rng.integers(-20, 20, (300, 1)).astype(np.float32)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids, gate, p = scores(z, "softmax", False, 4, st)
    want = np.exp(z.astype(np.float64) - z.max(1, keepdims=True))
    want /= want.sum(1, keepdims=True)
    assert int(st.item()) == 0
    assert (np.abs(p - want) <= 8 * p64.U32 * want).all()
    want = np.take_along_axis(want, ids, 1)
    assert (np.abs(gate - want) <= 8 * p64.U32 * want).all()
