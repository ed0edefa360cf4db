"""examples/moe_layer.py: microbatches in flight together, as a pipelined schedule has
them, get the gradients that each has alone.  Needs an MI355X.

Bound: the same kernels on the same inputs, so the same numbers but for the order in
which torch adds up a weight's gradient: below 1e-3 (one microbatch's ids or rows with
another's gradient are off by about 1)."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


@pytest.mark.parametrize("order", [(0, 1, 2), (2, 1, 0), (1, 2, 0)])
def test_forward_passes_before_the_first_backward_pass(order):
    spec = importlib.util.spec_from_file_location("moe_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    R, E, n_slot, k, T, H, F, n = 4, 16, 2, 2, 200, 64, 96, 3
    gen = torch.Generator(device="cuda").manual_seed(5)

    def rnd(*s):
        return torch.randn(*s, device="cuda", generator=gen)
    layer = m.Layer(R, E, n_slot, k, T, H, F)
    wg = (H ** -0.5 * rnd(E, H)).requires_grad_()
    w1 = (H ** -0.5 * rnd(E, 2 * F, H)).to(torch.bfloat16).requires_grad_()
    w2 = (F ** -0.5 * rnd(E, H, F)).to(torch.bfloat16).requires_grad_()
    xs = [rnd(T, H).to(torch.bfloat16).requires_grad_() for _ in range(n)]
    targets = [rnd(T, H) for _ in range(n)]

    def forward(i):
        gate, balance = m.Route.apply(xs[i].float() @ wg.t(), layer, 0.05)
        layer.make_plan()
        send = m.Dispatch.apply(xs[i], layer)
        out = m.Combine.apply(m.experts_bf16(send, layer, w1, w2), gate, layer)
        return ((out.float() - targets[i]) ** 2).mean() + balance.sum()

    def backward(i, loss):
        return torch.autograd.grad(loss, (xs[i], wg, w1, w2))
    alone = [backward(i, forward(i)) for i in range(n)]
    losses = [forward(i) for i in range(n)]
    together = {i: backward(i, losses[i]) for i in order}
    layer.check()
    for i in range(n):
        for a, b in zip(together[i], alone[i]):
            assert float((a.double() - b.double()).norm()) < 1e-3 * float(b.double().norm())
