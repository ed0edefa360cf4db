"""The router, its balance loss and its gradient on the GPU against the plain
64-bit implementation.  Needs an MI355X.

Tolerances, in units of u = 2^-24.  A score: the argument of exp is off by |z| u
at most (|z - c| <= 60 wherever a score counts), exp by 2 ulp, the sum over E by
its 16 serial and 9 tree steps, quotient and product by 3: under 100 u.  A sum of
n scores adds n u.  dlogits: the same roundings, twice, on terms whose magnitudes
the plain implementation sums; bf16 adds half an ulp of the result."""
import numpy as np
import pytest
import torch

import plain64 as p64

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

SCORE_U = 100 * p64.U32


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def logits(rng, T, E, bf16, spread=1.5, dead=0.0):
    z = (spread * rng.standard_normal((T, E))).astype(np.float32)
    if bf16:
        z = p64.bf16(z)
    z[rng.random((T, E)) < dead] = -np.inf
    return z


def apart(rng, z, r, bias, bf16):
    """Redraws the tokens whose selection hangs on a rounding."""
    for t in range(len(z)):
        for _ in range(50):
            key = p64.keys(z[t], r, bias)
            s = np.sort(key[key > -np.inf])
            gap = np.diff(s)
            close = ((gap > 0) & (gap < 3e-6)).any()
            if r["n_group"]:
                two = np.sort(key.reshape(r["n_group"], -1), axis=1)[:, -2:].sum(1)
                two = np.sort(two[two > -np.inf])
                close |= (np.diff(two) < 3e-6).any()
            if not close:
                break
            z[t] = logits(rng, 1, z.shape[1], bf16)[0]
    return z


def run_route(z, r, bf16, bias=None, mask=None, ld=None, stats=True, stream=None):
    T, E = z.shape
    ld = ld or E
    rows = np.full((T, ld), np.nan, np.float32)  # what lies between rows is not looked at
    rows[:, :E] = z
    lg = dev(p64.bf16_bits(rows).view(np.int16)) if bf16 else dev(rows)
    rt = uep.Router(E, r["k"], uep.ULTRAEP_SIGMOID if r["score"] == "sigmoid" else uep.ULTRAEP_SOFTMAX,
                    r["renorm"], r["n_group"], r["top_group"], r["scale"], r["seq_len"])
    n, f = rt.n_seg(T), torch.float32
    o = dict(topk=torch.full((T, r["k"]), 77, dtype=torch.int32, device="cuda"),
             gate=torch.full((T, r["k"]), 7., device="cuda"),
             counts=torch.full((n, E), 9, dtype=torch.int32, device="cuda"),
             prob_sum=torch.full((n, E), 9., dtype=f, device="cuda"),
             tokens=torch.full((n,), 9, dtype=torch.int32, device="cuda"))
    if not stats:
        o.update(counts=None, prob_sum=None, tokens=None)
    ws = torch.empty(uep.ultraep_route_ws_bytes(T, rt), dtype=torch.uint8, device="cuda").fill_(255)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    uep.ultraep_route(lg, T, ld, rt, None if bias is None else dev(bias),
                      None if mask is None else dev(mask.astype(np.uint8)), o["topk"], o["gate"],
                      o["counts"], o["prob_sum"], o["tokens"], ws if stats else None, st, stream=stream)
    torch.cuda.synchronize()
    return {k: None if v is None else v.cpu().numpy() for k, v in o.items()}, int(st.item()), lg, rt


def check_route(o, ref, stats=True):
    ids, gate, counts, psum, tokens = ref
    assert np.array_equal(o["topk"], ids)
    assert (np.abs(o["gate"] - gate) <= SCORE_U * gate + 1e-37).all()
    if stats:
        assert np.array_equal(o["counts"], counts) and np.array_equal(o["tokens"], tokens)
        assert (np.abs(o["prob_sum"] - psum) <= (SCORE_U + p64.U32 * tokens[:, None]) * psum + 1e-36).all()


def router(**kw):
    r = dict(E=16, k=3, score="softmax", renorm=True, n_group=0, top_group=0, scale=1.0, seq_len=0)
    return {**r, **kw}


CASES = [
    # E, k, T, score, renorm, n_group, top_group, seq_len, bf16, bias, ld
    (256, 8, 1, "sigmoid", True, 8, 4, 0, False, True, None),
    (256, 8, 67, "sigmoid", True, 8, 4, 16, False, True, None),
    (256, 8, 200, "sigmoid", False, 0, 0, 0, True, True, 264),
    (128, 8, 130, "softmax", True, 0, 0, 0, True, False, None),
    (128, 8, 33, "softmax", False, 4, 2, 7, False, False, 131),
    (72, 6, 70, "softmax", True, 8, 4, 0, True, False, None),
    (72, 6, 70, "sigmoid", False, 8, 3, 11, False, True, 73),
    (60, 4, 50, "sigmoid", True, 0, 0, 50, True, False, 61),
    (96, 12, 41, "softmax", False, 3, 2, 0, False, True, None),
    (16, 2, 512, "softmax", True, 0, 0, 100, False, False, None),
    (1, 1, 9, "softmax", False, 0, 0, 0, False, False, None),
    (2, 2, 17, "sigmoid", True, 1, 1, 1, False, False, None),
    (1024, 64, 20, "softmax", True, 0, 0, 0, False, False, 1024),
    (1024, 10, 20, "sigmoid", True, 64, 3, 3, True, True, None),
    (1020, 7, 21, "softmax", False, 34, 5, 0, False, False, None),
    (512, 12, 40, "sigmoid", True, 0, 0, 0, True, False, None),
    (384, 8, 35, "softmax", True, 8, 4, 9, True, False, 392),
    (5, 5, 30, "softmax", True, 0, 0, 0, True, False, None),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_route_loss_and_gradient(case):
    E, k, T, score, renorm, ng, tg, seq, bf16, with_bias, ld = case
    rng = np.random.default_rng(E * 1000 + T)
    r = router(E=E, k=k, score=score, renorm=renorm, n_group=ng, top_group=tg, seq_len=seq, scale=2.5)
    bias = (rng.integers(-200, 200, E) / 1024).astype(np.float32) if with_bias else None
    z = apart(rng, logits(rng, T, E, bf16), r, bias, bf16)
    mask = rng.random(T) > 0.2
    ref = p64.route(z, r, bias, mask)
    o, st, lg, rt = run_route(z, r, bf16, bias, mask, ld)
    assert st == 0
    check_route(o, ref)
    o2, st, _, _ = run_route(z, r, bf16, bias, mask, ld, stats=False)
    assert st == 0
    check_route(o2, ref, stats=False)
    # the same ids as the load count takes them
    cnt = torch.zeros(E, dtype=torch.int32, device="cuda")
    stw = torch.zeros(1, dtype=torch.int32, device="cuda")
    uep.ultraep_count(dev(o["topk"]), T, k, E, 1, cnt, stw)
    assert np.array_equal(cnt.cpu().numpy(), ref[2].sum(0))

    # the loss, with another rank's loads added
    n = len(ref[4])
    more = rng.integers(0, 50, (n, E)).astype(np.int32)
    ntok = ref[4].astype(np.int32) + 25
    counts = ref[2].astype(np.int32) + more
    loss, coef = torch.empty(1, device="cuda"), torch.empty((n, E), device="cuda")
    uep.ultraep_balance_loss(dev(counts), dev(ntok), dev(o["prob_sum"]), dev(o["tokens"]), n, rt, 0.01, loss, coef)
    rl, rc = p64.balance(counts, ntok, o["prob_sum"].astype(np.float64), ref[4], r, 0.01)
    got = coef.cpu().numpy()
    assert (np.abs(got - rc) <= 7 * p64.U32 * rc).all()   # alpha's own rounding, unit, c, f n, product, quotient
    assert abs(float(loss.item()) - rl) <= 8 * p64.U32 * rl

    # the gradient
    dg = rng.standard_normal((T, k)).astype(np.float32)
    dl = np.float32(1.7)
    w = (10 * rng.standard_normal((n, E))).astype(np.float32)
    out = torch.full_like(lg, 5)
    uep.ultraep_route_grad(lg, T, ld or E, rt, dev(mask.astype(np.uint8)), dev(o["topk"]), dev(dg), dev(w),
                           torch.tensor([dl], device="cuda"), out, stw)
    assert int(stw.item()) == 0
    got = out.cpu().numpy()
    if bf16:
        assert (got[:, E:] == 5).all()
        got = p64.from_bits(got.view(np.uint16))
    else:
        assert (got[:, E:] == 5).all()
    L = seq or T
    for t in range(T):
        if ref[0][t, 0] < 0:
            assert (got[t, :E] == 0).all()
            continue
        want, mag = p64.route_grad(z[t].astype(np.float64), ref[0][t], r, dg[t].astype(np.float64),
                                   float(dl) * w[t // L].astype(np.float64))
        tol = 2 * SCORE_U * mag + 1e-37 + (1.01 * p64.U16 * np.abs(want) if bf16 else 0)
        assert (np.abs(got[t, :E] - want) <= tol).all(), t


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True)])
@pytest.mark.parametrize("E,k,T,ld", [(3, 2, 2100, None), (16, 4, 2051, 20), (60, 4, 2100, None), (72, 6, 2500, 73),
                                      (96, 12, 2049, 96), (127, 8, 2100, 128), (128, 16, 4001, None), (136, 8, 6150, None),
                                      (192, 8, 6200, 200), (250, 5, 6145, None), (256, 8, 6200, 260)])
def test_gradient_of_many_tokens(E, k, T, ld, score, renorm, bf16):
    """Several tokens a wave: some masked, without ids, or of dead or very low logits."""
    rng = np.random.default_rng(E + T)
    r = router(E=E, k=k, score=score, renorm=renorm, scale=0.7, seq_len=1000)
    z = logits(rng, T, E, bf16, dead=0.05)
    look = np.unique(np.concatenate([[0, 1, 2, 3, T - 1], rng.integers(0, T, 40)]))
    z[look[5]] = -np.inf
    z[look[6::9]] = p64.bf16(z[look[6::9]] - 128)
    mask = rng.random(T) > 0.1
    ids = np.argsort(rng.random((T, E)), axis=1)[:, :k].astype(np.int32)
    few = rng.integers(0, k + 1, T)
    ids[np.arange(k) >= few[:, None]] = -1
    rows = np.full((T, ld or E), np.nan, np.float32)
    rows[:, :E] = z
    lg = dev(p64.bf16_bits(rows).view(np.int16)) if bf16 else dev(rows)
    dg = rng.standard_normal((T, k)).astype(np.float32)
    w = (10 * rng.standard_normal((-(-T // 1000), E))).astype(np.float32)
    rt = uep.Router(E, k, int(score == "sigmoid"), renorm, scale=0.7, seq_len=1000)
    out, st = torch.full_like(lg, 5), torch.zeros(1, dtype=torch.int32, device="cuda")
    uep.ultraep_route_grad(lg, T, ld or E, rt, dev(mask.astype(np.uint8)), dev(ids), dev(dg), dev(w), None, out, st)
    assert int(st.item()) == 0
    got = out.cpu().numpy()
    assert (got[:, E:] == 5).all()
    if bf16:
        got = p64.from_bits(got.view(np.uint16))
    # a few of them on their own: the same bits
    some, one = torch.from_numpy(look).cuda(), torch.full_like(lg[:len(look)], 5)
    rt.seq_len = 1
    uep.ultraep_route_grad(lg[some].contiguous(), len(look), ld or E, rt, dev(mask[look].astype(np.uint8)), dev(ids[look]),
                           dev(dg[look]), dev(w[look // 1000]), None, one, st)
    assert torch.equal(one.view(torch.int16), out[some].view(torch.int16)) and int(st.item()) == 0
    for t in look:
        if not mask[t] or few[t] == 0 or np.isneginf(z[t]).all():
            assert (got[t, :E] == 0).all(), t
            continue
        want, mag = p64.route_grad(z[t].astype(np.float64), ids[t], r, dg[t].astype(np.float64),
                                   w[t // 1000].astype(np.float64))
        tol = 2 * SCORE_U * mag + 1e-37 + (1.01 * p64.U16 * np.abs(want) if bf16 else 0)
        assert (np.abs(got[t, :E] - want) <= tol).all(), t


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_against_differences(score, renorm):
    """dlogits against central differences of the 64-bit objective."""
    rng = np.random.default_rng(8)
    T, E, k, h = 6, 20, 4, 1e-5
    r = router(E=E, k=k, score=score, renorm=renorm, scale=0.7)
    z = logits(rng, T, E, False, dead=0.1)
    ids = p64.route(z, r)[0]
    dg = rng.standard_normal((T, k)).astype(np.float32)
    w = rng.standard_normal((1, E)).astype(np.float32)
    rt = uep.Router(E, k, int(score == "sigmoid"), renorm, scale=0.7)
    out = torch.empty((T, E), device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    uep.ultraep_route_grad(dev(z), T, E, rt, None, dev(ids), dev(dg), dev(w), None, out, st)
    got = out.cpu().numpy()
    for t in range(T):
        z64, d, ww = z[t].astype(np.float64), dg[t].astype(np.float64), w[0].astype(np.float64)
        _, mag = p64.route_grad(z64, ids[t], r, d, ww)
        for e in range(E):
            if np.isneginf(z64[e]):
                assert got[t, e] == 0
                continue
            hi, lo = z64.copy(), z64.copy()
            hi[e] += h
            lo[e] -= h
            diff = (p64.objective(hi, ids[t], r, d, ww) - p64.objective(lo, ids[t], r, d, ww)) / (2 * h)
            assert abs(got[t, e] - diff) <= 2 * SCORE_U * mag[e] + 1e-8  # differences: h^2, 1e-16 / h


@pytest.mark.parametrize("E,k,score,ng,tg,bf16", [
    (256, 8, "sigmoid", 8, 4, False), (128, 8, "softmax", 0, 0, True), (72, 6, "softmax", 8, 3, True),
    (60, 16, "sigmoid", 0, 0, False), (384, 12, "softmax", 0, 0, False), (512, 8, "sigmoid", 16, 5, False),
    (640, 8, "softmax", 0, 0, True), (64, 17, "softmax", 0, 0, True)])
def test_many_tokens(E, k, score, ng, tg, bf16):
    """With and without statistics, and in calls of fewer tokens: the same ids, and
    equal sums for equal calls; a sample of the tokens against the plain form."""
    rng = np.random.default_rng(E)
    T = 4500
    r = router(E=E, k=k, score=score, n_group=ng, top_group=tg, seq_len=2100, scale=1.5)
    z = logits(rng, T, E, bf16, spread=1.0)
    z[:, :E // 5] += np.float32(2)   # neighbouring experts that most tokens choose among
    z = p64.bf16(z) if bf16 else z
    z[100:140] = z[100]              # and tokens in a row that are alike
    z[200:230] = 0.25                # or tie everywhere
    sample = np.r_[0:20, 95:105, 198:204, 4480:4500]
    z[sample] = apart(rng, z[sample], r, None, bf16)
    mask = rng.random(T) > 0.1
    o, st, lg, _ = run_route(z, r, bf16, mask=mask)
    assert st == 0
    ref = p64.route(z[sample], {**r, "seq_len": 0}, mask=mask[sample])
    check_route(dict(topk=o["topk"][sample], gate=o["gate"][sample]), ref, stats=False)
    seq = np.arange(T) // 2100
    for s in range(3):
        chosen = o["topk"][seq == s]
        assert np.array_equal(o["counts"][s], np.bincount(chosen[chosen >= 0], minlength=E))
        assert o["tokens"][s] == (chosen[:, 0] >= 0).sum() == mask[seq == s].sum()
    p = np.exp(z.astype(np.float64) - z.max(1, keepdims=True).astype(np.float64)) if score == "softmax" \
        else p64.sigmoid(z.astype(np.float64))
    p = p / p.sum(1, keepdims=True) * mask[:, None]
    psum = np.stack([p[seq == s].sum(0) for s in range(3)])
    assert (np.abs(o["prob_sum"] - psum) <= (SCORE_U + p64.U32 * 2100) * psum).all()
    again = run_route(z, r, bf16, mask=mask)[0]
    assert all(o[n].tobytes() == again[n].tobytes() for n in o)
    bare = run_route(z, r, bf16, mask=mask, stats=False)[0]
    few = [run_route(z[a:a + 1500], r, bf16, mask=mask[a:a + 1500], stats=False)[0] for a in (0, 1500, 3000)]
    for other in (bare, {n: np.concatenate([f[n] for f in few]) for n in ("topk", "gate")}):
        assert np.array_equal(other["topk"], o["topk"])
        assert (np.abs(other["gate"] - o["gate"]) <= 2 * SCORE_U * o["gate"]).all()


def test_ties_go_to_the_lower_id_and_group():
    z = np.zeros((3, 64), np.float32)
    z[1, 10:20] = 1.0
    z[1, 3] = -0.0
    z[2, 32:] = 2.0
    r = router(E=64, k=6)
    o, st, _, _ = run_route(z, r, False)
    assert st == 0
    assert o["topk"].tolist() == [[0, 1, 2, 3, 4, 5], [10, 11, 12, 13, 14, 15], [32, 33, 34, 35, 36, 37]]
    r = router(E=64, k=6, n_group=8, top_group=2)
    o, st, _, _ = run_route(z, r, False)
    assert o["topk"].tolist() == [[0, 1, 2, 3, 4, 5], [10, 11, 12, 13, 14, 15], [32, 33, 34, 35, 36, 37]]
    z = np.zeros((1, 64), np.float32)
    z[0, :3] = -0.0   # equal to +0
    assert run_route(z, router(E=64, k=2), False)[0]["topk"].tolist() == [[0, 1]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_infinite_and_lowest_logits(score):
    """Rows whose mask leaves fewer than k experts, one, or none; the type's
    lowest value is a number like others."""
    E, k = 40, 5
    low = np.finfo(np.float32).min
    z = np.full((8, E), -np.inf, np.float32)
    z[1, 7] = 0.5
    z[2, [3, 30, 31]] = [low, 1.0, low]
    z[3] = low
    z[4] = -200.0 - np.arange(E)
    z[5] = 150.0 + 0.5 * np.arange(E)
    z[6, [0, 39]] = -np.array([300.0, 300.5])
    z[7, 2:9] = 1.0
    for renorm in (True, False):
        for ng, tg in ((0, 0), (4, 2)):
            r = router(E=E, k=k, score=score, renorm=renorm, n_group=ng, top_group=tg)
            # keys in fp32: a sigmoid of these saturates, ties to the lower id
            ref_ids = np.array([p64.select(zz, r, None) if not (ng and score == "sigmoid") else
                                p64.select(np.where(np.isneginf(zz), zz, p64.sigmoid(zz.astype(np.float64))
                                                    .astype(np.float32)), {**r, "score": "softmax"}, None)
                                for zz in z])
            o, st, lg, rt = run_route(z, r, False)
            assert st == 0
            assert np.array_equal(o["topk"], ref_ids)
            assert np.isfinite(o["gate"]).all() and np.isfinite(o["prob_sum"]).all()
            for t in range(8):
                if ref_ids[t, 0] >= 0:
                    want = p64.gates(z[t], ref_ids[t], r)
                    # |z - c| reaches 3e38 where the score is 0, and 20 where it is not
                    assert (np.abs(o["gate"][t] - want) <= SCORE_U * want + 1e-37).all()
            assert int(o["tokens"][0]) == int((ref_ids[:, 0] >= 0).sum())
            dg = np.ones((8, k), np.float32)
            w = np.linspace(-1, 1, E).astype(np.float32)[None]
            out = torch.empty_like(lg)
            stw = torch.zeros(1, dtype=torch.int32, device="cuda")
            uep.ultraep_route_grad(lg, 8, E, rt, None, dev(ref_ids), dev(dg), dev(w), None, out, stw)
            got = out.cpu().numpy()
            assert int(stw.item()) == 0 and np.isfinite(got).all() and (got[np.isneginf(z)] == 0).all()
            for t in range(8):
                if ref_ids[t, 0] >= 0:
                    want, mag = p64.route_grad(z[t].astype(np.float64), ref_ids[t], r, dg[t].astype(np.float64),
                                               w[0].astype(np.float64))
                    assert (np.abs(got[t] - want) <= 2 * SCORE_U * mag + 1e-37).all()


@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("masked", [False, True])
def test_bad_logits(value, masked):
    """A NaN or +inf logit is reported and its token left out; in a masked token
    it is not looked at."""
    rng = np.random.default_rng(2)
    z = logits(rng, 20, 24, False)
    good = z.copy()
    z[11, 5] = value
    mask = np.ones(20, bool)
    mask[11] = False
    r = router(E=24, k=4)
    o, st, lg, rt = run_route(z, r, False, mask=mask if masked else None)
    assert st == (0 if masked else uep.ULTRAEP_EDATA)
    check_route(o, p64.route(good, r, None, mask))
    out = torch.empty_like(lg)
    stw = torch.zeros(1, dtype=torch.int32, device="cuda")
    uep.ultraep_route_grad(lg, 20, 24, rt, dev(mask.astype(np.uint8)) if masked else None, dev(o["topk"]),
                           torch.ones(20, 4, device="cuda"), None, None, out, stw)
    assert int(stw.item()) == (0 if masked else uep.ULTRAEP_EDATA)
    assert (out[11] == 0).all() and torch.isfinite(out).all()


@pytest.mark.parametrize("bad", [-2, 24, 1 << 30])
def test_bad_ids_in_the_gradient(bad):
    z = torch.randn(5, 24, device="cuda")
    ids = torch.tensor([[0, 1]] * 5, dtype=torch.int32, device="cuda")
    ids[3, 1] = bad
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty_like(z)
    uep.ultraep_route_grad(z, 5, 24, uep.Router(24, 2), None, ids, torch.ones(5, 2, device="cuda"), None, None, out, st)
    assert int(st.item()) == uep.ULTRAEP_EDATA and torch.isfinite(out).all()


def test_gradient_in_place_and_without_parts():
    """dlogits may be the logits' buffer; gates or loss alone; both left out is 0."""
    rng = np.random.default_rng(4)
    z = logits(rng, 50, 72, True)
    r = router(E=72, k=6, renorm=False)
    o, _, lg, rt = run_route(z, r, True)
    dg, w = torch.randn(50, 6, device="cuda"), torch.randn(1, 72, device="cuda")
    ids, st = dev(o["topk"]), torch.zeros(1, dtype=torch.int32, device="cuda")

    def grad(dgate, coef, out):
        uep.ultraep_route_grad(lg, 50, 72, rt, None, ids, dgate, coef, None, out, st)
        return out.clone()
    both = grad(dg, w, torch.empty_like(lg))
    a, b = grad(dg, None, torch.empty_like(lg)), grad(None, w, torch.empty_like(lg))
    zero = torch.zeros(1, device="cuda")
    out = torch.empty_like(lg)
    uep.ultraep_route_grad(lg, 50, 72, rt, None, ids, dg, w, zero, out, st)
    assert torch.equal(out, a)  # loss times 0
    f = [v.view(torch.bfloat16).double() for v in (both, a, b)]
    # three bf16 roundings, of the parts and of the sum
    assert ((f[0] - f[1] - f[2]).abs() <= 1.02 * p64.U16 * (f[0].abs() + f[1].abs() + f[2].abs()) + 1e-6).all()
    assert (grad(None, None, torch.empty_like(lg)).view(torch.bfloat16) == 0).all()
    assert torch.equal(grad(dg, w, lg), both)
    assert int(st.item()) == 0


def test_no_tokens():
    r = uep.Router(24, 4, seq_len=8)
    c, p, n = (torch.full(s, 3, dtype=d, device="cuda") for s, d in
               (((1, 24), torch.int32), ((1, 24), torch.float32), ((1,), torch.int32)))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(uep.ultraep_route_ws_bytes(0, r), dtype=torch.uint8, device="cuda")
    uep.ultraep_route(None, 0, 24, r, None, None, None, None, c, p, n, ws, st)
    assert (c == 0).all() and (p == 0).all() and (n == 0).all()
    loss, coef = torch.full((1,), 3., device="cuda"), torch.full((1, 24), 3., device="cuda")
    uep.ultraep_balance_loss(c, n, p, n, 1, r, 0.1, loss, coef)
    assert float(loss) == 0 and (coef == 0).all()
    loss.fill_(3)
    uep.ultraep_balance_loss(None, None, None, None, 0, r, 0.1, loss, None)
    assert float(loss) == 0
    uep.ultraep_route_grad(None, 0, 24, r, None, None, None, None, None, None, st)


def test_many_sequences_loss():
    """More coefficients than one pass of the loss's workgroup."""
    rng = np.random.default_rng(5)
    n, E = 700, 96
    r = router(E=E, k=4)
    c = rng.integers(0, 9, (n, E)).astype(np.int32)
    tok = rng.integers(0, 40, n).astype(np.int32)
    p = rng.random((n, E)).astype(np.float32)
    loss, coef = torch.empty(1, device="cuda"), torch.empty((n, E), device="cuda")
    uep.ultraep_balance_loss(dev(c), dev(tok), dev(p), dev(tok), n, uep.Router(E, 4), 0.02, loss, coef)
    rl, rc = p64.balance(c, tok, p.astype(np.float64), tok, r, 0.02)
    assert (np.abs(coef.cpu().numpy() - rc) <= 7 * p64.U32 * rc).all()
    assert abs(float(loss) - rl) <= 8 * p64.U32 * rl


def test_equal_calls_give_equal_bits_and_other_streams():
    rng = np.random.default_rng(6)
    z = logits(rng, 900, 128, False)
    r = router(E=128, k=8, seq_len=300)
    a = run_route(z, r, False)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = run_route(z, r, False, stream=s)[0]
    for n in a:
        assert a[n].tobytes() == b[n].tobytes(), n


def test_graph_replay():
    rng = np.random.default_rng(7)
    T, E, k = 300, 64, 4
    rt = uep.Router(E, k, uep.ULTRAEP_SIGMOID, seq_len=100)
    z = torch.empty(T, E, device="cuda")
    f, i = torch.float32, torch.int32
    o = [torch.empty(s, dtype=d, device="cuda") for s, d in
         (((T, k), i), ((T, k), f), ((3, E), i), ((3, E), f), ((3,), i))]
    ws = torch.empty(uep.ultraep_route_ws_bytes(T, rt), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=i, device="cuda")
    loss, coef, dz = torch.empty(1, device="cuda"), torch.empty(3, E, device="cuda"), torch.empty_like(z)

    def step():
        uep.ultraep_route(z, T, E, rt, None, None, *o, ws, st)
        uep.ultraep_balance_loss(o[2], o[4], o[3], o[4], 3, rt, 0.01, loss, coef)
        uep.ultraep_route_grad(z, T, E, rt, None, o[0], o[1], coef, loss, dz, st)
    z.copy_(torch.from_numpy(logits(rng, T, E, False)))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        z.copy_(torch.from_numpy(logits(rng, T, E, False)))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (*o, loss, coef, dz)]
        for t in (*o, loss, coef, dz):
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (*o, loss, coef, dz)))


def test_offsets_past_32_bits():
    """Logits of 5 GB: the last tokens' ids, gates and gradients."""
    T, E, ld, k = 5_000_003, 16, 256, 2
    z = torch.zeros(T, ld, device="cuda")
    tail = torch.randn(64, E, device="cuda")
    z[-64:, :E] = tail
    rt, st = uep.Router(E, k), torch.zeros(1, dtype=torch.int32, device="cuda")
    ids, gate = torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    uep.ultraep_route(z, T, ld, rt, None, None, ids, gate, None, None, None, None, st)
    r = router(E=E, k=k)
    check_route(dict(topk=ids[-64:].cpu().numpy(), gate=gate[-64:].cpu().numpy()), p64.route(tail.cpu().numpy(), r),
                stats=False)
    assert (ids[:-64] == torch.tensor([0, 1], device="cuda")).all()
    uep.ultraep_route_grad(z, T, ld, rt, None, ids, gate, None, None, z, st)
    one = torch.empty(64, E, device="cuda")
    uep.ultraep_route_grad(tail, 64, E, rt, None, ids[-64:].contiguous(), gate[-64:].contiguous(), None, None, one, st)
    assert torch.equal(z[-64:, :E], one) and int(st.item()) == 0
