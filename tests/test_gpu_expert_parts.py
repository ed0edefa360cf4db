"""The weights' gradient of few small weights, whose rows are summed in parts with a workspace
and joined by a second kernel: weights without rows.  Needs an MI355X."""
import numpy as np
import pytest
import torch

from test_gpu_expert_products import dev, dev16, normal, status

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
