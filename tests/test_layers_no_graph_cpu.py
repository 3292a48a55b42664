"""The plain calls return results without a graph: they refuse tensors whose gradient would be lost. (Without a GPU:
what is not refused goes on to ask for one.)"""
import types

import pytest
import torch

from paper_2212_11142_amd import layers


class Device(Exception):
    pass


@pytest.fixture(autouse=True)
def _stand_ins(monkeypatch):
    def none(*args, **kw):
        raise Device

    for name in ("NormBuffers", "GatedBuffers", "rotate_into"):
        monkeypatch.setattr(layers, name, none)


def calls():
    t = lambda grad: torch.zeros(3, 8, requires_grad=grad)               # noqa: E731
    return {"norm x": lambda g: layers.norm(None, t(g)),
            "norm weight": lambda g: layers.norm(None, t(False), weight=t(g)),
            "norm bias": lambda g: layers.norm(None, t(False), weight=t(False), bias=t(g)),
            "norm residual": lambda g: layers.norm(None, t(False), residual=t(g)),
            "rotate": lambda g: layers.rotate(types.SimpleNamespace(), None, t(g)),
            "gated x": lambda g: layers.gated(None, t(g), t(False), t(False)),
            "gated gate": lambda g: layers.gated(None, t(False), t(g), t(False)),
            "gated up": lambda g: layers.gated(None, t(False), t(False), t(g))}


@pytest.mark.parametrize("name", list(calls()))
def test_gradients_are_not_lost(name):
    f = calls()[name]
    with pytest.raises(ValueError, match="graph"):
        f(True)
    with pytest.raises(Device):
        f(False)
    with torch.no_grad(), pytest.raises(Device):
        f(True)
    with torch.inference_mode(), pytest.raises(Device):
        f(False)


def test_within_a_function():
    """Where autograd calls them, gradients are off."""
    class F(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            layers.gated(None, x, x, x)

    with pytest.raises(Device):
        F.apply(torch.zeros(3, 8, requires_grad=True))
