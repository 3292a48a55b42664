"""The Python binding of the layers without a GPU: tensors that only have a shape and an address, and a
library that records its calls; and what the layers' sources have to keep to."""
import ctypes as C
import os
import re
import types

import pytest
import torch

from paper_2212_11142_amd import gp, layers, seq

BF, F32 = torch.bfloat16, torch.float32
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2212_11142_amd", "csrc")


class Tensor:
    """What the binding asks of a CUDA tensor (index -1: of the host's)."""
    is_cuda = property(lambda self: self.index >= 0)

    def __init__(self, shape, dtype=BF, at=1 << 20, device=0, strides=None):
        self.shape, self.dtype, self.at, self.index, self.strides = torch.Size(shape), dtype, at, device, strides

    @property
    def device(self):
        return torch.device("cuda", self.index) if self.index >= 0 else torch.device("cpu")

    def stride(self):
        if self.strides:
            return self.strides
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s)

    def data_ptr(self):
        return self.at

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return self.strides is None


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


@pytest.fixture(autouse=True)
def _no_stream(monkeypatch):
    monkeypatch.setattr(layers, "_stream", lambda x: None)
    monkeypatch.setattr(seq, "_current_device", lambda: 0, raising=False)


# ------------------------------------------------------------------ norms
def norm(weight=F32, bias=True, **kw):
    n = layers.Norm(8, BF, weight=weight, bias=bias, **kw)
    n.lib = Library()
    t = lambda *s, dtype=BF: Tensor(s, dtype)                           # noqa: E731
    b = types.SimpleNamespace(norm=n, rows=3, device=0, shape=torch.Size((3, 8)), vector=torch.Size((8,)), out=t(3, 8),
                              sum=t(3, 8), stats=t(3, 2, dtype=F32), dx=t(3, 8), dweight=t(8, dtype=F32),
                              dbias=t(8, dtype=F32), workspace=None, workspace_bytes=0)
    return n, b


def test_norm():
    n, b = norm()
    x, w = Tensor((3, 8)), Tensor((8,), F32)
    layers.norm_into(n, x, b, weight=w, bias=w, residual=x)
    layers.norm_grad_into(n, x, x, b, weight=w)
    assert [c[0] for c in n.lib.calls] == ["gp_norm", "gp_norm_grad"]
    good = dict(weight=w, bias=w, residual=x)
    for kw in (dict(weight=None), dict(bias=None), dict(residual=None), dict(weight=Tensor((8,))), dict(weight=Tensor((9,), F32)),
               dict(weight=Tensor((8,), F32, device=1)), dict(weight=Tensor((8,), F32, strides=(2,))),
               dict(residual=Tensor((3, 8), F32)), dict(residual=Tensor((3, 8), strides=(8, 2)))):
        with pytest.raises(ValueError):
            layers.norm_into(n, x, b, **{**good, **kw})
    for y in (Tensor((2, 8)), Tensor((3, 9)), Tensor((3, 8), F32), Tensor((3, 8), device=1), Tensor((3, 8), device=-1),
              Tensor((3, 8), strides=(16, 2))):
        with pytest.raises(ValueError):
            layers.norm_into(n, y, b, **good)
        with pytest.raises(ValueError):
            layers.norm_grad_into(n, y, x, b, weight=w)
        with pytest.raises(ValueError):
            layers.norm_grad_into(n, x, y, b, weight=w)
        with pytest.raises(ValueError):
            layers.norm_grad_into(n, x, x, b, weight=w, dsum=y)
    with pytest.raises(ValueError):
        layers.norm_into(norm()[0], x, b, **good)
    with pytest.raises(ValueError):
        layers.norm_grad_into(norm()[0], x, x, b, weight=w)
    b.dx = None
    with pytest.raises(ValueError):
        layers.norm_grad_into(n, x, x, b, weight=w)


def test_norm_descriptions():
    for kw in (dict(eps=0.0), dict(weight=torch.float16)):
        with pytest.raises(gp.GPError):
            layers.Norm(8, BF, **kw)
    with pytest.raises(gp.GPError):
        layers.Norm(0, BF)
    with pytest.raises(ValueError):
        layers.Norm(8, BF, bias=True)
    with pytest.raises(TypeError):
        layers.Norm(8, torch.float64)


# ------------------------------------------------------------------ rotary positions
def rotary():
    r = layers.Rotary.__new__(layers.Rotary)
    r.dim, r.dtype, r.device, r.ref, r.lib = 64, BF, 0, None, Library()
    r.slots = layers._HeadSlots(r)
    return r


def test_rotary():
    r = rotary()
    x, p, s = Tensor((3, 4, 64)), Tensor((3,), torch.int32), Tensor((3,), torch.int64)
    k, cache = Tensor((3, 2, 64)), Tensor((9, 2, 64))
    layers.rotate_into(r, p, x, x)
    layers.append_into(r, p, s, x, k, k, x, cache, cache)
    assert [c[0] for c in r.lib.calls] == ["gp_rotate", "gp_rotate_append"]
    for y in (Tensor((3, 4, 60)), Tensor((3, 4, 64), F32), Tensor((3, 4, 64), device=1), Tensor((2, 4, 64)),
              Tensor((3, 4, 64), strides=(512, 128, 2))):
        with pytest.raises(ValueError):
            layers.rotate_into(r, p, x, y)
        with pytest.raises(ValueError):
            layers.rotate_into(r, p, y, x)
    for q in (Tensor((2,), torch.int32), Tensor((3,), torch.int64), Tensor((3,), torch.int32, device=-1),
              Tensor((3,), torch.int32, strides=(2,))):
        with pytest.raises(ValueError):
            layers.rotate_into(r, q, x, x)
    for args in ((p, p, x, k, k, x, cache, cache), (p, s, x, k, x, x, cache, cache), (p, s, x, k, k, k, cache, cache),
                 (p, s, x, k, k, x, cache, Tensor((8, 2, 64))), (p, s, x, k, k, x, Tensor((9, 4, 64)), cache)):
        with pytest.raises(ValueError):
            layers.append_into(r, *args)


def test_rotary_descriptions():
    for kw in (dict(base=0.0), dict(factor=-1.0), dict(original=100.0, near=2.0, far=2.0), dict(rotated=31),
               dict(angles=[1.0])):
        with pytest.raises(ValueError):
            layers.Rotary(64, BF, device=0, **kw)
    f = layers.frequencies(64, 10000.0, 4.0, original=8192, near=1.0, far=32.0)
    g = layers.frequencies(64, 10000.0)
    assert f[0] == g[0] and f[-1] == g[-1] / 4 and all(a <= b for a, b in zip(f, g))


# ------------------------------------------------------------------ gated block
def gated():
    t = layers.Gated(64, 72, BF)
    t.lib = Library()
    b = types.SimpleNamespace(gated=t, rows=3, device=0, x_shape=torch.Size((3, 64)), out_shape=torch.Size((3, 72)),
                              out=Tensor((3, 72)), dx=Tensor((3, 64)), dw_gate=Tensor((72, 64)), dw_up=Tensor((72, 64)),
                              workspace=None, workspace_bytes=0, slots=layers._MatrixSlots())
    return t, b


def test_gated():
    t, b = gated()
    x, w, d = Tensor((3, 64)), Tensor((72, 64)), Tensor((3, 72))
    layers.gated_into(t, x, w, w, b)
    layers.gated_grad_into(t, x, w, w, d, b)
    assert [c[0] for c in t.lib.calls] == ["gp_gated", "gp_gated_grad"]
    for y in (Tensor((3, 72)), Tensor((3, 64), F32), Tensor((3, 64), device=1), Tensor((3, 64), strides=(128, 2))):
        with pytest.raises(ValueError):
            layers.gated_into(t, y, w, w, b)
        with pytest.raises(ValueError):
            layers.gated_grad_into(t, y, w, w, d, b)
    for y in (Tensor((64, 72)), Tensor((72, 64), F32)):
        with pytest.raises(ValueError):
            layers.gated_into(t, x, y, w, b)
        with pytest.raises(ValueError):
            layers.gated_into(t, x, w, y, b)
        with pytest.raises(ValueError):
            layers.gated_grad_into(t, x, w, w, y, b)
    with pytest.raises(ValueError):
        layers.gated_into(gated()[0], x, w, w, b)
    b.dx = None
    with pytest.raises(ValueError):
        layers.gated_grad_into(t, x, w, w, d, b)


def test_gated_descriptions():
    for args, kw in (((60, 72, BF), {}), ((64, 0, BF), {}), ((64, 72, F32), {})):
        with pytest.raises(gp.GPError):
            layers.Gated(*args, **kw)
    with pytest.raises(ValueError):
        layers.Gated(64, 72, BF, activation="relu")
    with pytest.raises(gp.GPError):
        layers.Gated(64, 72, BF).grad_workspace_bytes(-1)


# ------------------------------------------------------------------ AdamW
def test_adamw_descriptions():
    p = [torch.zeros(3)]
    for args, kw in ((([],), {}), ((p,), {}), ((p,), dict(masters=[])), ((p,), dict(state_bits=16))):
        with pytest.raises(ValueError):
            layers.AdamW(*args, **kw)


def adamw_of(params, masters=None):
    """A state's marshalling alone, of host tensors."""
    o = layers.AdamW.__new__(layers.AdamW)
    o.params, o.masters, o.dtype, o.device = params, masters, params[0].dtype, -1
    o.shapes = [p.shape for p in params]
    o.tensors = (gp._AdamWTensor * len(params))()
    o._weights, o._at = params + (masters or []), None
    return o


def test_adamw_weights_share_no_memory():
    x = torch.zeros(64)
    a, b = x[:32], x[32:]
    adamw_of([b, a, torch.zeros(0), torch.zeros(0)])._update()
    for params in ([a, b, a], [x, a], [a, x[31:40]]):
        with pytest.raises(ValueError, match="share"):
            adamw_of(params)._update()
    h, w = torch.zeros(32, dtype=BF), torch.zeros(32)
    adamw_of([h], [w])._update()
    with pytest.raises(ValueError, match="share"):
        adamw_of([h, torch.zeros(32, dtype=BF)], [w, w])._update()
    with pytest.raises(ValueError, match="share"):
        adamw_of([w.view(BF)[:32]], [w])._update()


def test_adamw_weights_whose_layout_changes():
    """At the same address, too; and after a refusal the next call looks again."""
    p = torch.nn.Parameter(torch.zeros(4, 4))
    o = adamw_of([p])
    o._update()
    o._update()
    p.data = p.data.t()
    for _ in range(2):
        with pytest.raises(ValueError, match="contiguous"):
            o._update()
    p.data = torch.zeros(4, 4)
    o._update()
    assert o.tensors[0].param == p.data_ptr()


# ------------------------------------------------------------------ sources
@pytest.mark.parametrize("name", ["gated.hip", "norm.hip", "rotate.hip", "adamw.hip", "layer_dev.h"])
def test_no_vector_arithmetic_in_inline_assembly(name):
    """The results of a matrix or a transcendental instruction may be read a number of cycles later only, which
    the compiler counts for the instructions that it knows."""
    text = open(os.path.join(CSRC, name)).read()
    blocks = re.findall(r"\basm\s*(?:volatile)?\s*\(((?:[^()]|\([^()]*\))*)\)", text)
    assert blocks or name != "gated.hip"
    for b in blocks:
        code = "".join(re.findall(r'"((?:[^"\\]|\\.)*)"', b.split(":")[0]))
        assert not re.search(r"(?<![A-Za-z0-9_])v_[a-z]", code), (name, code)


def test_copies_wait_for_their_descriptor():
    """A buffer instruction reads scalar registers that a vector instruction may have written: 5 cycles have to lie
    between, which the compiler does not see to before inline assembly."""
    text = open(os.path.join(CSRC, "gated.hip")).read()
    blocks = re.findall(r"asm volatile\(((?:\s*\"[^\"]*\")+)", text)
    blocks = ["".join(re.findall(r'"([^"]*)"', b)).replace("\\n", "\n").replace("\\t", "\t") for b in blocks]
    blocks = [b for b in blocks if "buffer_load" in b]
    assert blocks
    for b in blocks:
        code = b.split("buffer_load")[0].split("\n")
        waits = sum(int(x.split()[1]) + 1 if x.split()[0] == "s_nop" else 1 for x in code if x.strip())
        assert waits >= 5, b


def tile_of(block, blocks, nm, nn):
    """gated.hip's mapping of blocks to tiles."""
    per, more, x = blocks // 8, blocks % 8, block % 8
    i = x * per + min(x, more) + block // 8
    group = i // (8 * nn)
    at = i - group * 8 * nn
    size = min(8, nm - group * 8)
    return group * 8 + at % size, at // size


@pytest.mark.parametrize("nm,nn", [(1, 1), (3, 5), (8, 4), (9, 7), (64, 32), (17, 1), (1, 40)])
def test_every_tile_has_its_block(nm, nn):
    seen = {tile_of(b, nm * nn, nm, nn) for b in range(nm * nn)}
    assert seen == {(m, n) for m in range(nm) for n in range(nn)}
