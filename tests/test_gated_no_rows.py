"""The gated block's gradient without rows."""
import pytest
import torch

from paper_2212_11142_amd import layers

pytestmark = pytest.mark.gpu

FP, BF = torch.float16, torch.bfloat16


@pytest.mark.parametrize("hidden", [72, 448, 456, 1368, 4096])
@pytest.mark.parametrize("dtype", [FP, BF])
def test_no_rows(hidden, dtype):
    """The weights' gradients of no rows are 0, at hidden sizes that are summed in parts too."""
    t = layers.Gated(64, hidden, dtype)
    b = layers.GatedBuffers(t, 0, grad=True)
    b.dw_gate.fill_(3), b.dw_up.fill_(3)
    x, d = torch.empty((0, 64), dtype=dtype, device="cuda"), torch.empty((0, hidden), dtype=dtype, device="cuda")
    w = torch.ones((hidden, 64), dtype=dtype, device="cuda")
    layers.gated_grad_into(t, x, w, w, d, b)
    assert not b.dw_gate.any() and not b.dw_up.any()
