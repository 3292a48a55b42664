"""The example's autograd Functions, on the CPU with stand-ins for the library's calls: nothing of a step stays behind
once its results are gone, not even until Python looks for cycles; and the gradient's call finds what the forward
call left."""
import gc
import os
import types

import pytest
import torch
from torch.multiprocessing.reductions import StorageWeakRef

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def ex(monkeypatch):
    monkeypatch.syspath_prepend(os.path.join(ROOT, "examples"))
    import in_context_surrogate
    gc.disable()
    yield in_context_surrogate
    gc.enable()


def buffers(**tensors):
    return types.SimpleNamespace(**tensors)


def norm(ex, monkeypatch, residual):
    made = []

    def make(norm, rows, residual=False, grad=False):
        made.append(buffers(out=torch.empty(rows, 4), sum=torch.empty(rows, 4) if residual else None,
                            stats=torch.empty(rows, 2), dx=torch.empty(rows, 4), dweight=torch.empty(4),
                            dbias=torch.empty(4)))
        return made[-1]

    def into(norm, x, b, weight, bias, residual):
        b.out.copy_(2 * x)
        b.stats.fill_(7)
        if residual is not None:
            b.sum.copy_(x + residual)

    def grad_into(norm, h, dout, b, weight, dsum):
        assert (b.stats == 7).all() and (h == (3 if residual else 1)).all()
        assert (dsum is not None) == residual
        b.dx.copy_(dout), b.dweight.fill_(1), b.dbias.fill_(1)

    monkeypatch.setattr(ex.layers, "NormBuffers", make)
    monkeypatch.setattr(ex.layers, "norm_into", into)
    monkeypatch.setattr(ex.layers, "norm_grad_into", grad_into)
    x, r = torch.ones(3, 4, requires_grad=True), torch.full((3, 4), 2.0, requires_grad=True)
    w, b = torch.ones(4, requires_grad=True), torch.ones(4, requires_grad=True)
    out = ex.Norm.apply(None, x, r if residual else None, w, b)
    return (out if residual else (out,)), ([x, r, w, b] if residual else [x, w, b]), made


def attend(ex, monkeypatch):
    made = []

    def make(att, grad):
        made.append(buffers(**{k: torch.empty(3, 2, 4) for k in ("out", "rest", "dq", "dk", "dv")}, lse=torch.empty(2, 3),
                            dtable=None))
        return made[-1]

    def into(att, q, k, v, b, table):
        b.out.fill_(5), b.rest.fill_(6), b.lse.fill_(7)

    def grad_into(att, q, k, v, dout, b, table):
        assert (b.out == 5).all() and (b.rest == 6).all() and (b.lse == 7).all()
        b.dq.copy_(dout), b.dk.copy_(dout), b.dv.copy_(dout)

    monkeypatch.setattr(ex.seq, "AttendBuffers", make)
    monkeypatch.setattr(ex.seq, "attend_into", into)
    monkeypatch.setattr(ex.seq, "attend_grad_into", grad_into)
    leaves = [torch.ones(3, 2, 4, requires_grad=True) for _ in range(3)]
    return (ex.Attend.apply(None, *leaves, None),), leaves, made


def logprob(ex, monkeypatch):
    made = []

    def make(rows, width, dtype, grad):
        made.append(buffers(logp=torch.empty(rows), entropy=torch.empty(rows), lse=torch.empty(rows),
                            norm=torch.empty(rows, 2), dlogits=torch.empty(rows, width)))
        return made[-1]

    def into(logits, targets, b):
        b.logp.fill_(5), b.entropy.fill_(6), b.norm.fill_(7)

    def grad_into(logits, targets, g_logp, g_entropy, b):
        assert (b.entropy == 6).all() and (b.norm == 7).all()
        b.dlogits.fill_(1)

    monkeypatch.setattr(ex.seq, "LogprobBuffers", make)
    monkeypatch.setattr(ex.seq, "logprob_into", into)
    monkeypatch.setattr(ex.seq, "logprob_grad_into", grad_into)
    x = torch.ones(3, 4, requires_grad=True)
    return ex.Logprob.apply(x, torch.zeros(3, dtype=torch.int64)), [x], made


CALLS = {"norm": lambda *a: norm(*a, residual=False), "norm of a sum": lambda *a: norm(*a, residual=True),
         "attend": attend, "logprob": logprob}


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("backward", [True, False])
def test_nothing_stays_behind(ex, monkeypatch, name, backward):
    outputs, leaves, made = CALLS[name](ex, monkeypatch)
    # (Nones: what the Function holds no more)
    kept = [t for t in vars(made[0]).values() if t is not None] + list(outputs)
    refs = [StorageWeakRef(t.untyped_storage()) for t in kept]
    if backward:
        torch.autograd.backward(outputs, [torch.ones_like(o) for o in outputs])
        assert all(x.grad is not None for x in leaves)
        leaves = [x.detach() for x in leaves]              # (gradients may be the buffers' own tensors)
    del outputs, kept, leaves
    made.clear()
    assert all(r.expired() for r in refs)


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["bias", "rotary"])
def test_training_keeps_no_memory(ex, order):
    """What is allocated after 3 steps and after 12: the weights and their gradients."""
    model = (ex.RotarySurrogate if order == "rotary" else ex.Surrogate)().cuda().bfloat16()
    held = []
    for steps in (3, 12):
        ex.train(model, steps, torch.Generator().manual_seed(1), runs=2, log=lambda line: None)
        torch.cuda.synchronize()
        held.append(torch.cuda.memory_allocated())
    assert held[0] == held[1]
