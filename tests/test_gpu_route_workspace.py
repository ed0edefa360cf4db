"""The router's statistics in a workspace sized for another batch, and its ends.
Needs an MI355X."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

F32, I32 = torch.float32, torch.int32


def statistics(z, r, ws):
    T, E = z.shape
    n = r.n_seg(T)
    o = [torch.full(s, 3, dtype=d, device="cuda") for s, d in
         (((T, r.k), I32), ((T, r.k), F32), ((n, E), I32), ((n, E), F32), ((n,), I32))]
    st = torch.zeros(1, dtype=I32, device="cuda")
    uep.ultraep_route(z, T, E, r, None, None, *o, ws, st)
    assert int(st.item()) == 0
    return o


@pytest.mark.parametrize("E,seq_len", [(256, 0), (256, 16384), (40, 0), (72, 5000)])
def test_workspace_of_a_larger_batch(E, seq_len):
    r = uep.Router(E, 4, seq_len=seq_len)
    z = torch.randn(16385, E, device="cuda")
    ws = torch.empty(uep.ultraep_route_ws_bytes(16385, r), dtype=torch.uint8, device="cuda")
    for T in (16384, 8192, 5001, 333, 16385):
        o = statistics(z[:T], r, ws)
        seq = torch.arange(T, device="cuda") // (seq_len or T)
        p = torch.softmax(z[:T].double(), 1)
        for s in range(r.n_seg(T)):
            mine = seq == s
            assert torch.equal(o[2][s].long(), torch.bincount(o[0][mine].reshape(-1).long(), minlength=E))
            assert int(o[4][s]) == int(mine.sum())
            want = p[mine].sum(0)
            # a score 100 roundings, a sum of T of them T more
            assert ((o[3][s] - want).abs() <= (100 + T) * 2.0 ** -24 * want).all()


@pytest.mark.parametrize("T,E,seq_len", [(16384, 256, 0), (16385, 256, 0), (9001, 64, 700), (20000, 128, 17000), (600, 16, 33)])
def test_partials_stay_in_the_workspace(T, E, seq_len):
    r = uep.Router(E, 2, seq_len=seq_len)
    n = uep.ultraep_route_ws_bytes(T, r)
    buf = torch.full((n + 8192,), 77, dtype=torch.uint8, device="cuda")
    z = torch.randn(T, E, device="cuda")
    o = statistics(z, r, buf[4096:4096 + n])
    assert int(o[4].sum()) == T and int(o[2].sum()) == 2 * T
    assert (buf[:4096] == 77).all() and (buf[4096 + n:] == 77).all()


@pytest.mark.parametrize("seq_len", [0, 8, 1 << 20, 1 << 40])
def test_no_tokens_of_long_sequences(seq_len):
    r = uep.Router(24, 4, seq_len=seq_len)
    c, p, n = (torch.full(s, 3, dtype=d, device="cuda") for s, d in (((1, 24), I32), ((1, 24), F32), ((1,), I32)))
    st = torch.zeros(1, dtype=I32, device="cuda")
    ws = torch.empty(uep.ultraep_route_ws_bytes(0, r), dtype=torch.uint8, device="cuda")
    uep.ultraep_route(None, 0, 24, r, None, None, None, None, c, p, n, ws, st)
    assert (c == 0).all() and (p == 0).all() and (n == 0).all() and int(st.item()) == 0
