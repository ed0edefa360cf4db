"""examples/moe_layer.py: the whole layer, forward, backward and served in 8-bit
integers, against torch.  Needs an MI355X.

Bounds: bf16 rows and products round to 2^-8 each, a handful of times (x, the two
products, the combined row, and their gradients): below 0.02.  8-bit rows and
weights have steps of max / 127: for normal values (max about 3.5 sigma) a rounding
error of 0.008 sigma each, four times, on top: below 0.05."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


@pytest.mark.parametrize("T,H,F", [(512, 256, 512), (333, 128, 208)])
def test_moe_layer_example(T, H, F):
    spec = importlib.util.spec_from_file_location("moe_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    bf16, int8, losses, grads = m.main(T, H, F, steps=30, verbose=False)
    assert bf16 < 0.02 and int8 < 0.05
    assert all(v < 0.02 for v in grads.values()), grads
    assert losses[-1] < losses[0] and losses[-1] >= 0.9
    assert torch.isfinite(torch.tensor(losses)).all()
