"""Selection biases that are no ordinary numbers, and groups of which one expert or
none can be chosen.  Needs an MI355X."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2606_04101_amd as uep

I32, F32 = torch.int32, torch.float32


def route(z, r, bias, stats):
    T, E = z.shape
    o = [torch.full((T, r.k), 7, dtype=I32, device="cuda"), torch.full((T, r.k), 7., device="cuda")]
    s = [torch.empty((1, E), dtype=I32, device="cuda"), torch.empty((1, E), device="cuda"),
         torch.empty(1, dtype=I32, device="cuda")] if stats else [None] * 3
    ws = torch.empty(uep.ultraep_route_ws_bytes(T, r), dtype=torch.uint8, device="cuda") if stats else None
    st = torch.zeros(1, dtype=I32, device="cuda")
    uep.ultraep_route(torch.from_numpy(z).cuda(), T, E, r, None if bias is None else torch.from_numpy(bias).cuda(), None,
                      *o, *s, ws, st)
    return o[0].cpu().numpy(), o[1].cpu().numpy(), int(st.item())


FORMS = [(E, T, stats) for E in (32, 256, 512) for T in (3, 3000) for stats in (False, True)]


@pytest.mark.parametrize("E,T,stats", FORMS)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups", [(0, 0), (8, 3)])
def test_nan_and_minus_infinity(E, T, stats, score, groups):
    """An expert whose bias is -inf or a NaN is not chosen; a NaN is reported."""
    rng = np.random.default_rng(E)
    z = np.stack([rng.permutation(E) for _ in range(T)]).astype(np.float32) / 64
    r = uep.Router(E, 4, uep.ULTRAEP_SIGMOID if score == "sigmoid" else uep.ULTRAEP_SOFTMAX, True, *groups)
    low = np.zeros(E, np.float32)
    low[[0, 1, 5, E - 1]] = -np.inf
    ids, gate, st = route(z, r, low, stats)
    assert st == 0 and (ids >= 0).all() and not np.isin(ids, [0, 1, 5, E - 1]).any()
    dead = np.where(np.isneginf(low), -np.inf, z).astype(np.float32)
    assert np.array_equal(ids, route(dead, r, np.zeros(E, np.float32), stats)[0])
    nan = np.where(np.isneginf(low), np.nan, low).astype(np.float32)
    got, g, st = route(z, r, nan, stats)
    assert st == uep.ULTRAEP_EDATA and np.array_equal(got, ids) and np.array_equal(g, gate)


@pytest.mark.parametrize("E,T,stats", FORMS)
@pytest.mark.parametrize("groups", [(0, 0), (8, 3)])
def test_infinite_bias_of_experts_out_of_service(E, T, stats, groups):
    """A logit of -inf stays one whatever the bias; +inf puts an expert in front."""
    rng = np.random.default_rng(E + 1)
    z = np.stack([rng.permutation(E) for _ in range(T)]).astype(np.float32) / 64
    bias = np.zeros(E, np.float32)
    bias[[1, 6, 9]] = np.inf
    z[:, [1, 6, E - 1]] = -np.inf
    for score in (uep.ULTRAEP_SOFTMAX, uep.ULTRAEP_SIGMOID):
        r = uep.Router(E, 4, score, True, *groups)
        ids, _, st = route(z, r, bias, stats)
        assert st == 0 and (ids[:, 0] == 9).all() and not np.isin(ids, [1, 6, E - 1]).any()
        big = np.zeros(E, np.float32)
        big[9] = 100   # in front as well
        assert np.array_equal(ids, route(z, r, big, stats)[0])


@pytest.mark.parametrize("E,T,stats", FORMS)
def test_a_group_of_one_choosable_expert_comes_last(E, T, stats):
    """Its sum of two is -inf, also where the one's key is +inf."""
    n, size = 8, E // 8
    z = np.full((T, E), 0.25, np.float32)
    z[:, 2 * size:3 * size] = -np.inf      # group 2: one expert left, its bias +inf
    z[:, 2 * size + 1] = 1.0
    z[:, 5 * size:6 * size] = -np.inf      # group 5: none
    bias = np.zeros(E, np.float32)
    bias[2 * size + 1] = np.inf
    bias[6 * size:] = 0.5                  # groups 6 and 7 are the best, then the lower ids
    for score in (uep.ULTRAEP_SOFTMAX, uep.ULTRAEP_SIGMOID):
        ids, _, st = route(z, uep.Router(E, 2 * size + 1, score, True, n, 3) if size < 8 else
                           uep.Router(E, 12, score, True, n, 3), bias, stats)
        want = (list(range(6 * size, E)) + list(range(size)))[:ids.shape[1]]
        assert st == 0 and (ids == np.array(want)).all()
    # best of all where only two groups have a sum: the lowest of those without one
    z[:, :2 * size] = -np.inf
    z[:, 3 * size:6 * size] = -np.inf
    ids, _, st = route(z, uep.Router(E, 2 * size + 1 if size < 8 else 12, uep.ULTRAEP_SOFTMAX, True, n, 3), bias, stats)
    want = list(range(6 * size, E)) + [-1]
    assert st == 0 and (ids == np.array(want[:ids.shape[1]])).all()


@pytest.mark.parametrize("T,stats", [(3, False), (3000, False), (3000, True)])
def test_one_group_is_no_groups(T, stats):
    """A sigmoid's keys are the logits there, also where the scores are all 1 or 0."""
    rng = np.random.default_rng(T)
    z = (np.stack([rng.permutation(64) for _ in range(T)]) + rng.choice([20, -200], (T, 1))).astype(np.float32)
    want = np.argsort(-z, axis=1)[:, :6]
    for groups in ((0, 0), (1, 1)):
        ids, _, st = route(z, uep.Router(64, 6, uep.ULTRAEP_SIGMOID, True, *groups), None, stats)
        assert st == 0 and np.array_equal(ids, want)
