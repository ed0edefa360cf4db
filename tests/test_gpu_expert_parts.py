"""The weights' gradient of few small weights, whose rows are summed in parts with a workspace
and joined by a second kernel: its binding, guards around outputs and workspace, captures,
streams, unsound lists, and weights without rows.  Needs an MI355X."""
import numpy as np
import pytest
import torch

from test_gpu_expert_binding import Declines
from test_gpu_expert_products import BAD_LISTS, dev, dev16, normal, status

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

M, N, K, G = 5000, 64, 72, 3
F32, BF16, U8, I32 = torch.float32, torch.bfloat16, torch.uint8, torch.int32


def workspace(M=M, N=N, K=K, n_w=G, guard=0):
    n = uep.ultraep_expert_weight_grad_ws_bytes(M, N, K, n_w)
    assert n > 16  # the rows are in parts
    return torch.full((n + 2 * guard,), 0x3F, dtype=U8, device="cuda")


def arguments(seed=0, type=F32, accumulate=False, sizes=(2500, 0, 2400), ws=None):
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)
    dw = torch.full((G, N, K), 0.5, dtype=type, device="cuda")
    return [dev16(normal(rng, M, N)), dev16(normal(rng, M, K)), M, N, K, dev(off), dev(np.array([2, 0, 1], np.int32)), 3, G,
            N * K, accumulate, dw, workspace() if ws is None else ws, status()]


@pytest.mark.parametrize("accumulate", [False, True])
def test_native_and_ctypes_halves_agree(accumulate, monkeypatch):
    a = arguments(accumulate=accumulate)
    uep.ultraep_expert_weight_grad(*a)
    torch.cuda.synchronize()
    first = a[11].clone()
    assert first.any()
    a[11].fill_(0.5)
    a[12].fill_(0xC1)
    monkeypatch.setattr(uep, "_native", Declines())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    uep.ultraep_expert_weight_grad(*a, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(a[11], first)


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("accumulate", [False, True])
def test_guards_around_outputs_and_workspace(type, accumulate):
    a = arguments(type=type, accumulate=accumulate)
    uep.ultraep_expert_weight_grad(*a)
    want = a[11].clone()
    buf = torch.full((G * N * K + 128,), 77.0, dtype=type, device="cuda")
    a[11] = buf[64:-64].view(G, N, K)
    a[11].fill_(0.5)
    ws = workspace(guard=256)
    a[12] = ws[256:-256]
    uep.ultraep_expert_weight_grad(*a)
    torch.cuda.synchronize()
    assert torch.equal(a[11], want)
    assert (buf[:64] == 77).all() and (buf[-64:] == 77).all()
    assert (ws[:256] == 0x3F).all() and (ws[-256:] == 0x3F).all()


def test_a_workspace_one_byte_short_is_refused():
    a = arguments()
    a[12] = a[12][:-1]
    with pytest.raises(uep.UltraEPError):
        uep.ultraep_expert_weight_grad(*a)


def test_captured_and_replayed():
    a = arguments()
    wants = []
    for src in (a[0].clone(), a[0].flip(0).contiguous()):
        a[0].copy_(src)
        uep.ultraep_expert_weight_grad(*a)
        wants.append((src, a[11].clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        uep.ultraep_expert_weight_grad(*a)
    for src, want in wants * 3:
        a[0].copy_(src)
        a[11].zero_()
        a[12].fill_(0x7F)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a[11], want)
        uep.ultraep_expert_weight_grad(*a)
        assert torch.equal(a[11], want)


def test_two_streams_at_once():
    sets = [arguments(seed=1), arguments(seed=2)]
    wants = []
    for a in sets:
        uep.ultraep_expert_weight_grad(*a)
        wants.append(a[11].clone())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for a in sets:
            a[11].zero_()
        torch.cuda.synchronize()
        for a, s in zip(sets, streams):
            for _ in range(3):
                uep.ultraep_expert_weight_grad(*a, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(a[11], w) for a, w in zip(sets, wants))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("off,of", BAD_LISTS)
def test_unsound_blocks_write_nothing(off, of, accumulate):
    """Neither the sums of the parts nor what the workspace holds reach dw."""
    a = arguments(accumulate=accumulate)
    assert max(off) <= M
    if max(off) == 21:  # (the list that ends behind its rows)
        off = off[:-1] + [M + 1]
    a[5], a[6] = dev(np.array(off, np.int64)), None if of is None else dev(np.array(of, np.int32))
    uep.ultraep_expert_weight_grad(*a)
    assert int(a[13].item()) == uep.ULTRAEP_EDATA and (a[11] == 0.5).all()


@pytest.mark.parametrize("type", [F32, BF16])
@pytest.mark.parametrize("parts", [True, False])
def test_a_weight_without_rows_stays_as_it_is(type, parts):
    """Accumulated: zeros of either sign, infinities and every NaN's bits."""
    a = arguments(type=type, accumulate=True)
    if not parts:
        a[12] = None
    words = torch.int32 if type == F32 else torch.int16
    g = torch.Generator(device="cuda").manual_seed(4)
    bits = torch.randint(-(1 << 15), 1 << 15, (G, N, K), generator=g, device="cuda")
    if type == F32:
        bits = bits * (1 << 16) + torch.randint(0, 1 << 16, (G, N, K), generator=g, device="cuda")
    bits = bits.to(words)
    bits[0, 0] = torch.iinfo(words).min  # -0
    a[11] = bits.view(type).clone()
    uep.ultraep_expert_weight_grad(*a)
    assert int(a[13].item()) == 0
    assert torch.equal(a[11][0].view(words), bits[0])
    assert not torch.equal(a[11][1].view(words), bits[1])


def test_the_most_rows():
    """2^31 - 1 rows in one block, all zero but for some from one end to the other: the steps
    of 64 that they take, 2^25, were counted by a sum past 2^31."""
    rows, N, K = (1 << 31) - 1, 8, 8
    dy, x = (torch.zeros(rows, n, dtype=BF16, device="cuda") for n in (N, K))
    at = torch.tensor([0, 63, 64, (1 << 30) - 1, (1 << 30) + 5, rows - 65, rows - 64, rows - 1], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(8)
    for t in (dy, x):
        t[at] = torch.randint(-3, 4, (len(at), 8), device="cuda", generator=g).to(BF16)  # exact sums
    dw, st = torch.full((N, K), 7.0, device="cuda"), status()
    uep.ultraep_expert_weight_grad(dy, x, rows, N, K, torch.tensor([0, rows], device="cuda"), None, 1, 1, N * K, False, dw,
                                   workspace(rows, N, K, 1), st)
    assert int(st.item()) == 0
    assert torch.equal(dw.double(), dy[at].double().t().contiguous() @ x[at].double())
