"""The binding of the experts' products: the native half takes the ordinary call, and
what it declines the ctypes half makes or refuses; outputs lie between guard bands;
calls on other streams, and captured and replayed ones, give the same.  Needs an
MI355X."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

M, N, K, G = 150, 48, 80, 3
F32, I32, I64, U8, BF16 = torch.float32, torch.int32, torch.int64, torch.uint8, torch.bfloat16
NAMES = ["matmul_bf16", "matmul_bf16_kept", "matmul_bf16_grad", "weight_grad", "weight_grad_parts", "quant_blocks",
         "matmul_fp8"]


def calls():
    """name -> (entry point, arguments in order, positions of outputs)."""
    g = torch.Generator(device="cuda").manual_seed(3)

    def rnd(*s, dtype=BF16):
        return torch.randn(*s, device="cuda", generator=g).to(dtype)

    def out(dtype, *s):
        return torch.zeros(*s, dtype=dtype, device="cuda")

    def e4m3(*s):
        return torch.randint(0x20, 0x40, s, dtype=U8, device="cuda", generator=g)
    st = out(I32, 1)
    off = torch.tensor([0, 70, 70, M], device="cuda")
    of = torch.tensor([2, 0, 1], dtype=I32, device="cuda")
    x, w = rnd(M, K), rnd(G, N, K)
    blocks = [off, of, G]
    ws = out(U8, uep.ultraep_expert_weight_grad_ws_bytes(M, N, K, G))
    scales = [out(U8, M, uep.scale_pitch(K)) + 127, out(U8, G, N, uep.scale_pitch(K)) + 125]
    return {
        "matmul_bf16": ("expert_matmul_bf16", [x, M, w, G, N * K, N, K, False, *blocks, uep.ULTRAEP_NO_ACT, None,
                                               out(F32, M, N), st], (13,)),
        "matmul_bf16_kept": ("expert_matmul_bf16", [x, M, w, G, N * K, N, K, False, *blocks, uep.ULTRAEP_SWIGLU,
                                                    out(BF16, M, N), out(BF16, M, N // 2), st], (12, 13)),
        "matmul_bf16_grad": ("expert_matmul_bf16", [x, M, w, G, N * K, N, K, True, *blocks, uep.ULTRAEP_SWIGLU_GRAD,
                                                    rnd(M, 2 * N), out(BF16, M, 2 * N), st], (13,)),
        "weight_grad": ("expert_weight_grad", [rnd(M, N), x, M, N, K, *blocks, G, N * K, False, out(F32, G, N, K), None, st],
                        (11,)),
        "weight_grad_parts": ("expert_weight_grad", [rnd(M, N), x, M, N, K, *blocks, G, N * K, False, out(BF16, G, N, K), ws,
                                                     st], (11,)),
        "quant_blocks": ("quant_blocks", [x, M, K, K, out(U8, M, K), K, out(U8, M, uep.scale_pitch(K))], (4, 6)),
        "matmul_fp8": ("expert_matmul_fp8", [e4m3(M, K), scales[0], M, e4m3(G, N, K), scales[1], G, N, K, *blocks, True,
                                             out(BF16, M, N // 2), st], (12,)),
    }


class Declines:
    def __getattr__(self, name):
        return lambda *a: None


@pytest.mark.parametrize("name", NAMES)
def test_native_and_ctypes_halves_agree(name, monkeypatch):
    entry, args, outs = calls()[name]
    f = getattr(uep, "ultraep_" + entry)
    assert getattr(uep._load_native(), entry)(*args, None) == 0
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
    entry, args, _ = calls()[name]
    native = getattr(uep._load_native(), entry)
    for i, t in enumerate(args):
        if not isinstance(t, torch.Tensor) or (entry == "expert_weight_grad" and i == 12):  # (the library's to check)
            continue
        for bad in (t.reshape(-1)[:-1].contiguous(), t.cpu(), t.to(torch.float64 if t.element_size() < 8 else F32),
                    torch.stack([t, t], -1)[..., 0]):
            if bad.numel() == t.numel() and bad.is_contiguous() and bad.is_cuda and bad.dtype == t.dtype:
                continue
            assert native(*args[:i], bad, *args[i + 1:], None) is None, (i, bad.shape, bad.dtype)
            with pytest.raises((ValueError, uep.UltraEPError)):
                getattr(uep, "ultraep_" + entry)(*args[:i], bad, *args[i + 1:])
    assert native(*args) is None  # no stream argument
    assert native(*args, "0") is None


def test_a_short_workspace_is_refused():
    _, args, _ = calls()["weight_grad_parts"]
    args[12] = torch.empty(15, dtype=U8, device="cuda")
    with pytest.raises(uep.UltraEPError):
        uep.ultraep_expert_weight_grad(*args)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("name", NAMES)
def test_guard_bands(name, native, monkeypatch):
    """Outputs in the middle of larger buffers, 64 bytes from their ends' guards."""
    entry, args, outs = calls()[name]
    if not native:
        monkeypatch.setattr(uep, "_native", Declines())
    f = getattr(uep, "ultraep_" + entry)
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


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name):
    """A graph of the call replayed over changing inputs, with eager work between."""
    entry, args, outs = calls()[name]
    f = getattr(uep, "ultraep_" + entry)
    first = 0 if entry != "expert_matmul_fp8" else 3
    other = args[first].flip(0).contiguous()
    wants = []
    for src in (args[first].clone(), other):
        args[first].copy_(src)
        f(*args)
        wants.append((src, [args[i].clone() for i in outs]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(*args)
    for src, want in wants * 3:
        args[first].copy_(src)
        for i in outs:
            args[i].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(args[i], t) for i, t in zip(outs, want))
        f(*args)  # eagerly too, between the replays
        assert all(torch.equal(args[i], t) for i, t in zip(outs, want))


def test_two_streams_at_once():
    """Calls interleaved on two streams, each with its own outputs and workspaces."""
    sets = [calls(), calls()]
    for name in NAMES:
        for entry, args, _ in (s[name] for s in sets):
            getattr(uep, "ultraep_" + entry)(*args)
    torch.cuda.synchronize()
    wants = [{n: [s[n][1][i].clone() for i in s[n][2]] for n in NAMES} for s in sets]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for name in NAMES:
            for s, stream in zip(sets, streams):
                entry, args, outs = s[name]
                for i in outs:
                    args[i].zero_()
            torch.cuda.synchronize()
            for s, stream in zip(sets, streams):
                entry, args, outs = s[name]
                with torch.cuda.stream(stream):
                    getattr(uep, "ultraep_" + entry)(*args)
            torch.cuda.synchronize()
    for s, want in zip(sets, wants):
        for n in NAMES:
            assert all(torch.equal(s[n][1][i], t) for i, t in zip(s[n][2], want[n]))


def test_float8_tensors_are_taken():
    _, args, _ = calls()["matmul_fp8"]
    uep.ultraep_expert_matmul_fp8(*args)
    want = args[12].clone()
    e4m3, e8m0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
    for i, t in ((0, e4m3), (1, e8m0), (3, e4m3), (4, e8m0)):
        args[i] = args[i].view(t)
    args[12] = torch.zeros_like(args[12])
    uep.ultraep_expert_matmul_fp8(*args)
    assert torch.equal(args[12], want)
