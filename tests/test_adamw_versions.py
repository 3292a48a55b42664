"""A step of AdamW counts as a change of its weights in place: what autograd saved of them before is refused by a
backward pass after it."""
import pytest
import torch

from paper_2212_11142_amd import gp, layers


def stepped(monkeypatch, masters):
    """A state of host tensors whose library does nothing, and a step of it."""
    params = [torch.nn.Parameter(torch.ones(3, dtype=torch.bfloat16 if masters else torch.float32)) for _ in range(2)]
    o = layers.AdamW.__new__(layers.AdamW)
    o.params, o.masters = params, [torch.ones(3) for _ in params] if masters else None
    o.dtype = o.grad_dtype = params[0].dtype
    o.device, o.shapes = -1, [p.shape for p in params]
    o.tensors, o.pointers = (gp._AdamWTensor * 2)(), gp.C.c_void_p * 2
    o._weights, o._at, o.struct = params + (o.masters or []), None, gp._AdamW()
    o.lib = type("Library", (), {"gp_adamw": staticmethod(lambda *a: 0)})
    monkeypatch.setattr(layers, "_stream", lambda x: None)
    monkeypatch.setattr(layers, "_call", lambda device, f, args: f(*args))
    return o


@pytest.mark.parametrize("masters", [False, True])
def test_steps_are_counted(monkeypatch, masters):
    o = stepped(monkeypatch, masters)
    before = [w._version for w in o._weights]
    a, b = o.params
    y = (a * a).sum()
    z = (b * b).sum()
    layers.adamw_into(o, [torch.ones_like(a), None], lr=0.1, step=1)
    # (a weight without a gradient is left as it is)
    moved = [w._version - v for w, v in zip(o._weights, before)]
    assert moved == [1, 0] * (2 if masters else 1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    z.backward()


def test_weights_without_a_counter(monkeypatch):
    """Tensors of inference mode have none."""
    o = stepped(monkeypatch, False)
    with torch.inference_mode():
        o.params = o._weights = [torch.ones(3), torch.ones(3)]
        layers.adamw_into(o, [torch.ones(3), torch.ones(3)], lr=0.1, step=1)
    layers.adamw_into(o, [torch.ones(3), torch.ones(3)], lr=0.1, step=2)


@pytest.mark.gpu
def test_on_the_device():
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    opt = layers.AdamW([p])
    y = (p * p).sum()
    layers.adamw_into(opt, [torch.ones_like(p)], lr=0.1, step=1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    (p * p).sum().backward()
    assert p.grad is not None
