"""What AdamW's binding looks at on each call, without a GPU."""
import pytest
import torch

from paper_2212_11142_amd import gp, layers

BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32


def adamw_of(params, masters=None):
    """A state's marshalling alone, of host tensors."""
    o = layers.AdamW.__new__(layers.AdamW)
    o.params, o.masters, o.dtype, o.device = params, masters, params[0].dtype, -1
    o.shapes = [p.shape for p in params]
    o.tensors = (gp._AdamWTensor * len(params))()
    o._weights, o._at = params + (masters or []), None
    return o


@pytest.mark.parametrize("change", [lambda x: x[:2], lambda x: x.view(FP), lambda x: x.view(2, 8),
                                    lambda x: x.view(F32), lambda x: x[:0]])
def test_weights_that_change_at_the_same_address(change):
    """A shorter, a re-typed and a reshaped view of a weight's own memory; after a refusal the next call looks
    again, and what was there before is taken again."""
    p = torch.nn.Parameter(torch.zeros(4, 4, dtype=BF))
    o = adamw_of([torch.zeros(3, dtype=BF), p])
    o._update()
    keep = p.data
    p.data = change(keep)
    assert p.numel() == 0 or p.data_ptr() == keep.data_ptr()
    for _ in range(2):
        with pytest.raises(ValueError, match="weight 1"):
            o._update()
    p.data = keep
    o._update()
    o._update()


@pytest.mark.parametrize("change", [lambda x: x[:2], lambda x: x.view(torch.int32), lambda x: x.view(2, 8)])
def test_master_copies_that_change_at_the_same_address(change):
    w = torch.zeros(4, 4)
    o = adamw_of([torch.zeros(4, 4, dtype=BF)], [w])
    o._update()
    keep = w.data
    w.data = change(keep)
    for _ in range(2):
        with pytest.raises(ValueError, match="master copy 0"):
            o._update()
    w.data = keep
    o._update()


@pytest.mark.parametrize("name", ["m", "v", "scales", "m_all", "v_all", "scales_all"])
def test_states_are_copied_into(name):
    """The library has their addresses: a tensor put in their place would not be used."""
    o = layers.AdamW.__new__(layers.AdamW)
    with pytest.raises(AttributeError):
        setattr(o, name, torch.zeros(3))
