"""The operators around the balancing path, without a GPU: the plain 64-bit
implementations against differences and closed forms, the workspace sizes, and
what the C ABI and the binding refuse before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_04101_amd as uep
import plain64 as p64

E_ = uep.ULTRAEP_EINVAL


def router(**kw):
    r = dict(E=16, k=3, score="softmax", renorm=True, n_group=0, top_group=0, scale=1.0, seq_len=0)
    return {**r, **kw}


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dead", [0, 2])
def test_gradient_formula_against_differences(score, renorm, dead):
    """Central differences in 64 bits: error about h^2 / 6 of the third derivative
    (below 10 of the objective's scale here) plus rounding 1e-16 / h."""
    rng = np.random.default_rng(3)
    r = router(score=score, renorm=renorm, scale=2.5)
    h = 1e-5
    for _ in range(5):
        z = rng.standard_normal(16) * 2
        z[rng.permutation(16)[:dead]] = -np.inf
        ids = p64.select(z.astype(np.float32), r, None)
        dg, w = rng.standard_normal(3), rng.standard_normal(16)
        got, _ = p64.route_grad(z, ids, r, dg, w)
        for e in range(16):
            if np.isneginf(z[e]):
                assert got[e] == 0
                continue
            hi, lo = z.copy(), z.copy()
            hi[e] += h
            lo[e] -= h
            d = (p64.objective(hi, ids, r, dg, w) - p64.objective(lo, ids, r, dg, w)) / (2 * h)
            assert abs(d - got[e]) < 1e-8


def test_balance_loss_of_an_even_load_is_alpha():
    """Every expert equally often and equally probable: loss = alpha."""
    r = router(k=2)
    counts = np.full((3, 16), 5)
    tok = np.full(3, 40)
    loss, coef = p64.balance(counts, tok, np.full((3, 16), 40 / 16), tok, r, 0.01)
    assert abs(loss - 0.01) < 1e-15 and coef.shape == (3, 16)


def test_route_workspace_bytes():
    r = uep.Router(256, 8)
    assert uep.ultraep_route_ws_bytes(0, r) >= 4
    assert uep.ultraep_route_ws_bytes(1, r) >= 4
    assert uep.ultraep_route_ws_bytes(4096, r) > 0
    assert uep.ultraep_route_ws_bytes(-1, r) == 0
    assert uep.ultraep_route_ws_bytes((1 << 23) + 1, r) == 0
    assert uep.ultraep_route_ws_bytes(8, uep.Router(1025, 8)) == 0


BAD_ROUTERS = [uep.Router(0, 1), uep.Router(1025, 1), uep.Router(16, 0), uep.Router(16, 17),
               uep.Router(128, 65), uep.Router(16, 2, score=2), uep.Router(16, 2, n_group=3, top_group=1),
               uep.Router(16, 2, n_group=4, top_group=5), uep.Router(16, 2, n_group=4, top_group=0),
               uep.Router(16, 2, n_group=16, top_group=4), uep.Router(16, 5, n_group=4, top_group=1),
               uep.Router(16, 2, n_group=0, top_group=1), uep.Router(16, 2, seq_len=-1),
               uep.Router(16, 2, scale=float("inf")), uep.Router(16, 2, scale=float("nan")),
               uep.Router(512, 2, n_group=128, top_group=4), uep.Router(16, 2, renorm=2)]


def test_bad_routers_are_refused():
    L, p = uep.lib(), ctypes.c_void_p(4096)  # never dereferenced: validation fails first
    for r in BAD_ROUTERS:
        b = ctypes.byref(r)
        assert L.ultraep_route(p, 0, 8, 1024, b, None, None, p, p, None, None, None, None, 0, p, None) == E_
        assert L.ultraep_balance_loss(p, p, p, p, 1, b, 0.1, p, p, None) == E_
        assert L.ultraep_route_grad(p, 0, 8, 1024, b, None, p, None, None, None, p, p, None) == E_


def test_bad_arguments_are_refused():
    L, p, odd = uep.lib(), ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 2)
    r = ctypes.byref(uep.Router(16, 2))

    def route(logits=p, type=0, T=8, ld=16, topk=p, gate=p, stats=(None, None, None), ws=None, n=0, status=p):
        return L.ultraep_route(logits, type, T, ld, r, None, None, topk, gate, *stats, ws, n, status, None)
    for kw in [dict(type=2), dict(T=-1), dict(T=(1 << 23) + 1), dict(ld=15), dict(ld=(1 << 20) + 1),
               dict(logits=None), dict(logits=odd), dict(topk=None), dict(gate=None), dict(status=None),
               dict(stats=(p, None, None)), dict(stats=(None, p, p)), dict(stats=(p, p, p)),
               dict(stats=(p, p, p), ws=p, n=3), dict(stats=(p, p, p), ws=odd, n=1 << 20)]:
        assert route(**kw) == E_, kw
    assert route(T=0, logits=None, topk=None, gate=None) == uep.ULTRAEP_OK  # nothing to do

    for a in [(None, p, p, p, 1), (p, None, p, p, 1), (p, p, None, p, 1), (p, p, p, None, 1), (p, p, p, p, -1)]:
        assert L.ultraep_balance_loss(*a, r, 0.1, p, p, None) == E_
    assert L.ultraep_balance_loss(p, p, p, p, 1, r, float("nan"), p, p, None) == E_
    assert L.ultraep_balance_loss(p, p, p, p, 1, r, 0.1, None, p, None) == E_
    assert L.ultraep_balance_loss(p, p, p, p, 1, r, 0.1, p, None, None) == E_

    def grad(logits=p, type=0, T=8, ld=16, topk=p, out=p, status=p):
        return L.ultraep_route_grad(logits, type, T, ld, r, None, topk, None, None, None, out, status, None)
    for kw in [dict(type=-1), dict(T=-1), dict(ld=8), dict(logits=None), dict(topk=None), dict(out=None),
               dict(out=odd), dict(status=None)]:
        assert grad(**kw) == E_, kw
    assert grad(T=0) == uep.ULTRAEP_OK

    def cg(dout=p, y=p, n_rows=16, gate=p, rows=p, T=8, k=2, H=16, n=p, dy=ctypes.c_void_p(8192), dg=p, st=p):
        return L.ultraep_combine_grad(dout, y, n_rows, gate, rows, T, k, H, n, dy, dg, st, None)
    for kw in [dict(H=12), dict(H=0), dict(k=0), dict(k=65), dict(T=-1), dict(n_rows=-1), dict(n_rows=1 << 31),
               dict(T=1 << 30), dict(dout=None), dict(dout=odd), dict(y=None), dict(y=odd), dict(gate=None),
               dict(rows=None), dict(n=None), dict(dy=None), dict(dy=odd), dict(dy=p), dict(dg=None),
               dict(st=None)]:
        assert cg(**kw) == E_, kw
    assert cg(T=0, n_rows=0) == uep.ULTRAEP_OK

    def quant(x=p, type=1, rows=4, K=16, ld=16, q=p, ldq=16, scale=p):
        return L.ultraep_quant_rows(x, type, rows, K, ld, q, ldq, scale, None)
    for kw in [dict(type=2), dict(rows=-1), dict(rows=1 << 31), dict(K=0), dict(K=12), dict(ld=8), dict(ld=20),
               dict(ld=(1 << 20) + 8), dict(ldq=8), dict(ldq=24), dict(ldq=(1 << 20) + 16), dict(x=None),
               dict(x=odd), dict(q=None), dict(q=odd), dict(scale=None)]:
        assert quant(**kw) == E_, kw
    assert quant(rows=0) == uep.ULTRAEP_OK

    def mm(xq=p, xs=p, M=4, wq=p, ws=p, n_w=2, N=16, K=32, off=p, of=None, n=2, act=0, y=p, type=1, st=p):
        return L.ultraep_expert_matmul(xq, xs, M, wq, ws, n_w, N, K, off, of, n, act, y, type, st, None)
    for kw in [dict(M=-1), dict(M=1 << 31), dict(M=1 << 30, N=256), dict(n_w=0), dict(N=0), dict(N=12), dict(N=(1 << 20) + 8),
               dict(N=8, act=1), dict(act=2), dict(K=0), dict(K=24), dict(K=(1 << 16) + 16), dict(n=0),
               dict(n=2049), dict(type=3), dict(xq=None), dict(xq=odd), dict(xs=None), dict(wq=None),
               dict(wq=odd), dict(ws=None), dict(off=None), dict(y=None), dict(y=odd), dict(st=None)]:
        assert mm(**kw) == E_, kw
    assert mm(M=0) == uep.ULTRAEP_OK


def t(n, dtype=torch.int32):
    return torch.zeros(n, dtype=dtype)


def test_binding_refuses_small_or_wrong_tensors():
    T, E, k, H = 6, 16, 3, 16
    r, f, b = uep.Router(E, k, seq_len=2), torch.float32, torch.bfloat16
    ok = dict(logits=t(T * E, f), bias=None, mask=None, topk=t(T * k), gate=t(T * k, f), counts=t(3 * E),
              prob_sum=t(3 * E, f), tokens=t(3), ws=None, status=t(1))
    for name, bad in [("logits", t(T * E - 1, f)), ("logits", t(T * E, torch.float16)), ("logits", t(T * E)),
                      ("logits", t(T * E, torch.float64)), ("bias", t(E - 1, f)), ("mask", t(T)),
                      ("topk", t(T * k - 1)), ("gate", t(T * k, b)), ("counts", t(3 * E - 1)),
                      ("prob_sum", t(2 * E, f)), ("tokens", t(2)), ("status", None)]:
        a = {**ok, name: bad}
        with pytest.raises(ValueError, match=name):
            uep.ultraep_route(a["logits"], T, E, r, *list(a.values())[1:])
    with pytest.raises(ValueError, match="logits"):  # the last row's end, rows apart
        uep.ultraep_route(t(T * E, f), T, E + 1, r, *list(ok.values())[1:])
    bl = dict(counts=t(3 * E), load_tokens=t(3), prob_sum=t(3 * E, f), tokens=t(3))
    for name, bad in [("counts", t(3 * E - 1)), ("load_tokens", t(2)), ("prob_sum", t(3 * E, b)), ("tokens", None)]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_balance_loss(*{**bl, name: bad}.values(), 3, r, 0.1, t(1, f), t(3 * E, f))
    with pytest.raises(ValueError, match="coef"):
        uep.ultraep_balance_loss(*bl.values(), 3, r, 0.1, t(1, f), t(3 * E - 1, f))
    g = dict(mask=None, topk=t(T * k), dgate=t(T * k, f), coef=t(3 * E, f), dloss=t(1, f), dlogits=t(T * E, f),
             status=t(1))
    for name, bad in [("topk", None), ("dgate", t(T * k - 1, f)), ("coef", t(3 * E - 1, f)), ("dloss", t(0, f)),
                      ("dlogits", t(T * E - 1, f)), ("dlogits", t(T * E, b)), ("mask", t(T - 1, torch.uint8))]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_route_grad(t(T * E, f), T, E, r, *{**g, name: bad}.values())
    c = dict(dout=t(T * H, b), y=t(T * k * H, b), n_rows=T * k, gate=t(T * k, f), row_of_slot=t(T * k), T=T, k=k,
             H=H, n_routed=t(1, torch.int64), dy=t(T * k * H, b), dgate=t(T * k, f), status=t(1))
    for name, bad in [("dout", t(T * H - 1, b)), ("y", t(T * k * H - 1, b)), ("gate", None),
                      ("row_of_slot", t(1)), ("n_routed", t(1)), ("dy", t(T * k * H, f)), ("dgate", t(1, f))]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_combine_grad(*{**c, name: bad}.values())
    for name, bad in [("x", t(4 * 24 - 9, b)), ("x", t(4 * 24, torch.float16)), ("q", t(4 * 32 - 1, torch.int8)),
                      ("q", t(4 * 32)), ("scale", t(3, f))]:
        a = {**dict(x=t(3 * 32 + 24, b), q=t(4 * 32, torch.int8), scale=t(4, f)), name: bad}
        with pytest.raises(ValueError, match=name):
            uep.ultraep_quant_rows(a["x"], 4, 24, 32, a["q"], 32, a["scale"])
    i8 = torch.int8
    m = dict(xq=t(4 * 32, i8), x_scale=t(4, f), M=4, wq=t(2 * 16 * 32, i8), w_scale=t(32, f), n_w=2, N=16, K=32,
             block_off=t(3, torch.int64), block_w=None, n_block=2, act=1, y=t(4 * 8, b), status=t(1))
    for name, bad in [("xq", t(4 * 32 - 1, i8)), ("x_scale", t(3, f)), ("wq", t(2 * 16 * 32 - 1, i8)),
                      ("w_scale", t(31, f)), ("block_off", t(2, torch.int64)), ("block_off", t(3)),
                      ("block_w", t(1)), ("y", t(4 * 8 - 1, b)), ("y", t(4 * 8, torch.float16)), ("status", t(0))]:
        with pytest.raises(ValueError, match=name):
            uep.ultraep_expert_matmul(*{**m, name: bad}.values())


def test_native_half_declines_host_tensors():
    n, f = uep._load_native(), torch.float32
    r = uep.Router(16, 2)
    assert n.route(t(16, f), 1, 16, r, None, None, t(2), t(2, f), None, None, None, None, t(1), 0) is None
    assert n.balance_loss(t(16), t(1), t(16, f), t(1), 1, r, 0.1, t(1, f), t(16, f), 0) is None
    assert n.balance_loss(t(16), t(1), t(16, f), t(1), 1, r, "0.1", t(1, f), t(16, f), 0) is None
    assert n.quant_rows(t(16, f), 1, 16, 16, t(16, torch.int8), 16, t(1, f), 0) is None
    assert n.route(t(16, f), 1, 16, object(), None, None, t(2), t(2, f), None, None, None, None, t(1), 0) is None


def test_quantisation_is_within_half_a_step():
    x = np.random.default_rng(1).standard_normal((20, 64)).astype(np.float32)
    q, s = p64.quant_rows(x)
    assert np.abs(q).max() == 127
    # half a step, and the roundings of x * (127 / a), of at most 127
    assert (np.abs(x - q * s[:, None].astype(np.float64)) <= s[:, None] * (0.5 + 127 * 4 * p64.U32)).all()
