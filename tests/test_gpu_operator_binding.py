"""The binding of the operators around the balancing path: the native half takes
the ordinary call, and what it declines the ctypes half makes or refuses; outputs
lie between guard bands that stay as they are.  Needs an MI355X."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

T, E, k, H, M, N, K, G = 37, 40, 3, 72, 50, 48, 80, 3
F32, I32, I64, I8, BF16 = torch.float32, torch.int32, torch.int64, torch.int8, torch.bfloat16
V = T * k


def calls():
    """name -> (arguments in order, positions of outputs)."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def rnd(*s, dtype=F32):
        return torch.randn(*s, device="cuda", generator=g).to(dtype)

    def out(dtype, *s):
        return torch.zeros(*s, dtype=dtype, device="cuda")
    r = uep.Router(E, k, uep.ULTRAEP_SIGMOID, seq_len=10)
    n = r.n_seg(T)
    z = rnd(T, E)
    ids = z.topk(k, 1).indices.to(I32).contiguous()
    st = out(I32, 1)
    i8 = (rnd(M, K) * 30).clamp(-127, 127).to(I8)
    w8 = (rnd(G, N, K) * 30).clamp(-127, 127).to(I8)
    off = torch.tensor([0, 20, 20, M], device="cuda")
    pos = torch.rand(n, E, device="cuda", generator=g)
    return {
        "route": ([z, T, E, r, rnd(E), torch.ones(T, dtype=torch.uint8, device="cuda"), out(I32, T, k), out(F32, T, k),
                   out(I32, n, E), out(F32, n, E), out(I32, n), out(torch.uint8, uep.ultraep_route_ws_bytes(T, r)), st],
                  (6, 7, 8, 9, 10)),
        "balance_loss": ([out(I32, n, E) + 2, out(I32, n) + 10, pos, out(I32, n) + 10, n, r, 0.25, out(F32, 1),
                          out(F32, n, E)], (7, 8)),
        "route_grad": ([z, T, E, r, None, ids, rnd(T, k), rnd(n, E), rnd(1), out(F32, T, E), st], (9,)),
        "combine_grad": ([rnd(T, H, dtype=BF16), rnd(V, H, dtype=BF16), V, rnd(T, k),
                          torch.arange(V, dtype=I32, device="cuda"), T, k, H, torch.tensor([V], device="cuda"),
                          out(BF16, V, H), out(F32, T, k), st], (9, 10)),
        "quant_rows": ([rnd(M, K, dtype=BF16), M, K, K, out(I8, M, K), K, out(F32, M)], (4, 6)),
        "expert_matmul": ([i8, rnd(M), M, w8, rnd(G, N), G, N, K, off, torch.tensor([2, 0, 1], dtype=I32, device="cuda"),
                           G, True, out(BF16, M, N // 2), st], (12,)),
    }


NAMES = ["route", "balance_loss", "route_grad", "combine_grad", "quant_rows", "expert_matmul"]


class Declines:
    def __getattr__(self, name):
        return lambda *a: None


@pytest.mark.parametrize("name", NAMES)
def test_native_and_ctypes_halves_agree(name, monkeypatch):
    args, outs = calls()[name]
    native, f = uep._load_native(), getattr(uep, "ultraep_" + name)
    assert getattr(native, name)(*args, None) == 0
    torch.cuda.synchronize()
    first = [args[i].clone() for i in outs]
    assert any(t.any() for t in first)
    for i in outs:
        args[i].zero_()
    monkeypatch.setattr(uep, "_native", Declines())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    assert f(*args, stream=s) == 0
    torch.cuda.synchronize()
    assert all(torch.equal(args[i], t) for i, t in zip(outs, first))


@pytest.mark.parametrize("name", NAMES)
def test_what_the_native_half_declines(name):
    """A buffer one element short, of another width, on the host, or not contiguous."""
    args, _ = calls()[name]
    native = getattr(uep._load_native(), name)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor) or (name == "route" and i == 11):  # (the workspace is the library's to check)
            continue
        for bad in (t.reshape(-1)[:-1].contiguous(), t.cpu(), t.to(torch.float64 if t.element_size() < 8 else F32),
                    torch.stack([t, t], -1)[..., 0]):
            if bad.numel() == t.numel() and bad.is_contiguous() and bad.is_cuda and bad.dtype == t.dtype:
                continue
            assert native(*args[:i], bad, *args[i + 1:], None) is None, (i, bad.shape, bad.dtype)
            with pytest.raises((ValueError, uep.UltraEPError)):
                getattr(uep, "ultraep_" + name)(*args[:i], bad, *args[i + 1:])
    assert native(*args) is None  # no stream argument
    assert native(*args, "0") is None


def test_library_refusals_through_the_native_half():
    args, _ = calls()["route"]
    one = uep.Router(E, k)  # one sequence, of several workgroups
    full = torch.empty(uep.ultraep_route_ws_bytes(T, one), dtype=torch.uint8, device="cuda")
    assert uep.ultraep_route(*args[:3], one, *args[4:11], full, args[12]) == 0
    for bad in (full[:-1].contiguous(), None):
        with pytest.raises(uep.UltraEPError):
            uep.ultraep_route(*args[:3], one, *args[4:11], bad, args[12])
    with pytest.raises(uep.UltraEPError):
        uep.ultraep_route(*args[:3], uep.Router(E, k, n_group=7, top_group=1), *args[4:])
    args, _ = calls()["quant_rows"]
    with pytest.raises(uep.UltraEPError):
        uep.ultraep_quant_rows(args[0], M, K - 4, K, *args[4:])


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_guard_bands(name, native, monkeypatch):
    """Outputs in the middle of larger buffers, 64 bytes from their ends' guards."""
    args, outs = calls()[name]
    if not native:
        monkeypatch.setattr(uep, "_native", Declines())
    f = getattr(uep, "ultraep_" + name)
    f(*args)
    torch.cuda.synchronize()
    want = [args[i].clone() for i in outs]
    bufs = []
    for i in outs:
        t = args[i]
        pad = 64 // t.element_size()
        buf = torch.full((t.numel() + 2 * pad,), 77, dtype=t.dtype, device="cuda")
        args[i] = buf[pad:pad + t.numel()].view(t.shape)
        bufs.append((buf, pad))
    f(*args)
    torch.cuda.synchronize()
    for i, w, (buf, pad) in zip(outs, want, bufs):
        assert torch.equal(args[i], w)
        assert (buf[:pad] == 77).all() and (buf[-pad:] == 77).all()


def test_bf16_forms():
    """bf16 logits and results as bfloat16 and as raw 16-bit integers."""
    args, _ = calls()["route_grad"]
    z = args[0].to(BF16)
    o = [torch.zeros_like(z), torch.zeros(T, E, dtype=torch.int16, device="cuda")]
    uep.ultraep_route_grad(z, *args[1:9], o[0], args[10])
    uep.ultraep_route_grad(z.view(torch.int16), *args[1:9], o[1], args[10])
    assert torch.equal(o[0].view(torch.int16), o[1]) and o[1].any()
    with pytest.raises(ValueError, match="dlogits"):
        uep.ultraep_route_grad(z, *args[1:9], args[9], args[10])
    assert np.isfinite(o[0].float().cpu().numpy()).all()
