"""An in-context surrogate: a small attention model that learns from many tuning runs to
predict the outcome of a candidate configuration from a run's observations.

Each run is one document of a packed batch: its observations (configuration and outcome),
which every row of the run reads (prefix), then the configurations whose outcome is asked
for. The order of the rows enters as a learned bias by buckets of their distance, scores are
capped, and the answer is a distribution over bins of the outcome, trained by the log
probability of the bin that came out and a little entropy. Afterwards the trained model
scores a large batch of candidates against one run's observations (every candidate reads all
of them), and one candidate at a time from the same keys and values.

With --order rotary the order enters as rotary positions of the queries and keys instead, the layers
have norms with weights and a gated feed-forward block, and AdamW makes the steps.

    python examples/in_context_surrogate.py [--steps 400] [--order rotary]

Runs are drawn from a Gaussian-process prior over unit-cube configurations.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2212_11142_amd import layers, seq  # noqa: E402

DIM, HEADS, KV_HEADS, HEAD, LAYERS, BINS, PARAMS = 256, 8, 4, 64, 3, 128, 2
GATED = 2 * DIM + 128                       # hidden values of the gated block
CAP, BUCKETS = 30.0, seq.log_buckets(16, 128, two_sided=True)
LOW, HIGH = -4.0, 4.0                       # range of the bins (standardised outcomes)


# ------------------------------------------------------------------ the operators in autograd
# (A context keeps a call's buffers without its outputs: those belong to the graph, whose node belongs to them and
# has the context, a cycle that would keep each step's buffers. What the gradient reads of them is saved.)
class Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, att, q, k, v, table):
        bufs = seq.AttendBuffers(att, grad=True)
        seq.attend_into(att, q, k, v, bufs, table=table)
        out, bufs.out = bufs.out, None
        ctx.att, ctx.bufs = att, bufs
        ctx.save_for_backward(q, k, v, table, out)
        return out

    @staticmethod
    def backward(ctx, dout):
        b = ctx.bufs
        q, k, v, table, b.out = ctx.saved_tensors
        seq.attend_grad_into(ctx.att, q, k, v, dout.contiguous(), b, table=table)
        b.out = None
        return None, b.dq, b.dk, b.dv, b.dtable


class Logprob(torch.autograd.Function):
    """(log probability of the targets, entropy) of rows of logits."""

    @staticmethod
    def forward(ctx, logits, targets):
        bufs = seq.LogprobBuffers(*logits.shape, logits.dtype, grad=True)
        seq.logprob_into(logits, targets, bufs)
        logp, entropy, bufs.logp, bufs.entropy = bufs.logp, bufs.entropy, None, None
        ctx.bufs = bufs
        ctx.save_for_backward(logits, targets, entropy)
        return logp, entropy

    @staticmethod
    def backward(ctx, g_logp, g_entropy):
        b = ctx.bufs
        logits, targets, b.entropy = ctx.saved_tensors
        seq.logprob_grad_into(logits, targets, g_logp.contiguous(), g_entropy.contiguous(), b)
        b.entropy = None
        return b.dlogits, None


class Norm(torch.autograd.Function):
    """The norm of x, or of x + residual and that sum."""

    @staticmethod
    def forward(ctx, norm, x, residual, weight, bias):
        bufs = layers.NormBuffers(norm, x.shape[0], residual=residual is not None, grad=True)
        layers.norm_into(norm, x, bufs, weight=weight, bias=bias, residual=residual)
        out, total, bufs.out, bufs.sum = bufs.out, bufs.sum, None, None
        ctx.norm, ctx.bufs = norm, bufs
        ctx.save_for_backward(x if residual is None else total, weight)
        return out if residual is None else (out, total)

    @staticmethod
    def backward(ctx, dout, dsum=None):
        h, weight = ctx.saved_tensors
        b = ctx.bufs
        layers.norm_grad_into(ctx.norm, h, dout.contiguous(), b, weight=weight,
                              dsum=None if dsum is None else dsum.contiguous())
        return None, b.dx, b.dx if ctx.needs_input_grad[2] else None, b.dweight, b.dbias


class Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rotary, positions, x):
        ctx.rotary, ctx.positions = rotary, positions
        return layers.rotate(rotary, positions, x)

    @staticmethod
    def backward(ctx, dout):
        return None, None, layers.rotate(ctx.rotary, ctx.positions, dout.contiguous(), inverse=True)


class Gated(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gated, x, w_gate, w_up):
        ctx.gated = gated
        ctx.save_for_backward(x, w_gate, w_up)
        return layers.gated(gated, x, w_gate, w_up)

    @staticmethod
    def backward(ctx, dout):
        x, w_gate, w_up = ctx.saved_tensors
        b = layers.GatedBuffers(ctx.gated, x.shape[0], grad=True)
        layers.gated_grad_into(ctx.gated, x, w_gate, w_up, dout.contiguous(), b)
        return None, b.dx, b.dw_gate, b.dw_up


# ------------------------------------------------------------------ model
def norm(x):
    return x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)


class Layer(torch.nn.Module):
    def __init__(self):
        super().__init__()
        self.qkv = torch.nn.Linear(DIM, (HEADS + 2 * KV_HEADS) * HEAD, bias=False)
        self.out = torch.nn.Linear(HEADS * HEAD, DIM, bias=False)
        self.up = torch.nn.Linear(DIM, 4 * DIM)
        self.down = torch.nn.Linear(4 * DIM, DIM)
        self.table = torch.nn.Parameter(torch.zeros(HEADS, BUCKETS.count))

    def keys_values(self, x):
        y = self.qkv(norm(x)).view(-1, HEADS + 2 * KV_HEADS, HEAD)
        return y[:, :HEADS], y[:, HEADS:HEADS + KV_HEADS], y[:, HEADS + KV_HEADS:]

    def rest(self, x, y):
        x = x + self.out(y.reshape(-1, HEADS * HEAD))
        return x + self.down(torch.nn.functional.gelu(self.up(norm(x))))

    def forward(self, x, att):
        q, k, v = self.keys_values(x)
        return self.rest(x, Attend.apply(att, q, k, v, self.table))


class RotaryLayer(torch.nn.Module):
    """x, and what the layers before add to it, kept apart until a norm adds them up."""

    def __init__(self, dtype=torch.bfloat16):
        super().__init__()
        self.qkv = torch.nn.Linear(DIM, (HEADS + 2 * KV_HEADS) * HEAD, bias=False)
        self.out = torch.nn.Linear(HEADS * HEAD, DIM, bias=False)
        self.gate = torch.nn.Linear(DIM, GATED, bias=False)
        self.up = torch.nn.Linear(DIM, GATED, bias=False)
        self.down = torch.nn.Linear(GATED, DIM, bias=False)
        self.scale = torch.nn.ParameterList(torch.nn.Parameter(torch.ones(DIM)) for _ in range(2))
        self.shift = torch.nn.ParameterList(torch.nn.Parameter(torch.zeros(DIM)) for _ in range(2))
        self.norm = layers.Norm(DIM, dtype, weight=dtype, bias=True)
        self.gated = layers.Gated(DIM, GATED, dtype, activation="silu")
        self.rotary = layers.Rotary(HEAD, dtype, base=1000.0)

    def heads(self, x, added):
        """The heads of a row's queries, keys and values, and the row."""
        y, x = Norm.apply(self.norm, x, added, self.scale[0], self.shift[0])
        return self.qkv(y).view(-1, HEADS + 2 * KV_HEADS, HEAD), x

    def rest(self, x, y):
        y, x = Norm.apply(self.norm, x, self.out(y.reshape(-1, HEADS * HEAD)), self.scale[1], self.shift[1])
        return x, self.down(Gated.apply(self.gated, y, self.gate.weight, self.up.weight))

    def forward(self, x, added, att, positions):
        y, x = self.heads(x, added)
        qk = Rotate.apply(self.rotary, positions, y[:, :HEADS + KV_HEADS])
        return self.rest(x, Attend.apply(att, qk[:, :HEADS], qk[:, HEADS:], y[:, HEADS + KV_HEADS:], None))


class Surrogate(torch.nn.Module):
    order = "bias"

    def __init__(self):
        super().__init__()
        self.config = torch.nn.Linear(PARAMS * 16, DIM)
        self.outcome = torch.nn.Linear(2, DIM)               # the value, and whether known
        self.layers = torch.nn.ModuleList(Layer() for _ in range(LAYERS))
        self.head = torch.nn.Linear(DIM, BINS)

    def embed(self, configs, outcomes, known):
        waves = configs[:, :, None] * (0.5 * math.pi * torch.arange(1, 9, device="cuda"))
        x = torch.cat([waves.sin(), waves.cos()], 2).flatten(1)
        y = torch.stack([torch.where(known, outcomes, 0.0), known.float()], 1)
        return self.config(x.bfloat16()) + self.outcome(y.bfloat16())

    def forward(self, configs, outcomes, known, att):
        x = self.embed(configs, outcomes, known)
        for layer in self.layers:
            x = layer(x, att)
        return self.head(norm(x))


class RotarySurrogate(Surrogate):
    order = "rotary"

    def __init__(self):
        super().__init__()
        self.layers = torch.nn.ModuleList(RotaryLayer() for _ in range(LAYERS))
        self.scale = torch.nn.Parameter(torch.ones(DIM))
        self.last = layers.Norm(DIM, torch.bfloat16, weight=torch.bfloat16)

    def answers(self, x, added):
        return self.head(Norm.apply(self.last, x + added, None, self.scale, None))

    def forward(self, configs, outcomes, known, att):
        x = self.embed(configs, outcomes, known)
        added, positions = torch.zeros_like(x), layers.positions(att.docs)
        for layer in self.layers:
            x, added = layer(x, added, att, positions)
        return self.answers(x, added)


def bin_of(y):
    return ((y - LOW) / (HIGH - LOW) * BINS).long().clamp(0, BINS - 1)


# ------------------------------------------------------------------ data
def draw_runs(count, observed, asked, gen):
    """`count` runs from a GP prior: configurations [rows, PARAMS], outcomes [rows], and per
    run its (observed, asked) numbers of rows."""
    xs, ys, sizes = [], [], []
    for _ in range(count):
        n = int(torch.randint(observed // 2, observed + 1, (1,), generator=gen))
        m = int(torch.randint(asked // 2, asked + 1, (1,), generator=gen))
        x = torch.rand((n + m, PARAMS), generator=gen)
        scale = 0.4 + 0.4 * torch.rand((PARAMS,), generator=gen)
        r = torch.cdist((x / scale).double(), (x / scale).double())
        k = (1 + math.sqrt(5) * r + 5 / 3 * r * r) * torch.exp(-math.sqrt(5) * r)
        l = torch.linalg.cholesky(k + 1e-4 * torch.eye(n + m, dtype=torch.float64))
        y = (l @ torch.randn((n + m,), generator=gen, dtype=torch.float64)).float()
        xs.append(x)
        ys.append((y - y[:n].mean()) / (y[:n].std() + 1e-3))
        sizes.append((n, m))
    return torch.cat(xs).cuda(), torch.cat(ys).cuda(), sizes


def batch_of(xs, ys, sizes):
    """What a packed batch needs beside its rows: which outcomes are known, the targets (-1
    where they are), and the documents with their prefixes."""
    known = torch.cat([torch.arange(n + m) < n for n, m in sizes]).cuda()
    docs = seq.Documents([n + m for n, m in sizes], prefix=[n for n, _ in sizes])
    return known, torch.where(known, -1, bin_of(ys)), docs


def attention(docs, causal=True, buckets=BUCKETS):
    return seq.Attention(docs, HEADS, KV_HEADS, HEAD, torch.bfloat16, causal=causal, cap=CAP,
                         buckets=buckets)


def train(model, steps, gen, runs=16, observed=64, asked=64, log=print):
    master = [p.detach().float().clone() for p in model.parameters()]   # fp32 weights
    rotary = model.order == "rotary"
    if rotary:
        own = layers.AdamW([p.detach() for p in model.parameters()], masters=master)
    else:
        opt = torch.optim.Adam(master, lr=1e-3)
    losses = []
    for step in range(steps):
        rate = 1e-3 * min(1.0, (step + 1) / 50)
        xs, ys, sizes = draw_runs(runs, observed, asked, gen)
        known, target, docs = batch_of(xs, ys, sizes)
        logits = model(xs, ys, known, attention(docs, buckets=None if rotary else BUCKETS))
        logp, entropy = Logprob.apply(logits, target)
        rows = (target >= 0).sum()
        # rows without a target have logp 0 and take no part; a little entropy keeps the
        # distribution from closing early
        loss = -(logp.sum() + 0.01 * entropy[target >= 0].sum()) / rows
        model.zero_grad()
        loss.backward()
        if rotary:
            layers.adamw_into(own, [p.grad for p in model.parameters()], lr=rate, step=step + 1)
        else:
            for group in opt.param_groups:
                group["lr"] = rate
            for w, p in zip(master, model.parameters()):
                w.grad = p.grad.float()
            opt.step()
            with torch.no_grad():
                for w, p in zip(master, model.parameters()):
                    p.copy_(w)
        losses.append(-(logp.sum() / rows).item())
        if step % 50 == 0 or step == steps - 1:
            log(f"step {step:4d}: -log p of the outcome's bin {losses[-1]:.3f} "
                f"(uniform {math.log(BINS):.3f})")
    return losses


# ------------------------------------------------------------------ answers
@torch.no_grad()
def answer(model, x_obs, y_obs, candidates, one_by_one=0):
    """Logits of every candidate given a run's observations. The observations read one
    another, the candidates read them; both in one call per layer, or for the first
    `one_by_one` candidates one row per call from the observations' keys and values."""
    n, m = x_obs.shape[0], candidates.shape[0]
    obs = model.embed(x_obs, y_obs, torch.ones(n, dtype=torch.bool, device="cuda"))
    cand = model.embed(candidates, torch.zeros(m, device="cuda"),
                       torch.zeros(m, dtype=torch.bool, device="cuda"))
    att_obs = attention(seq.Documents([n], prefix=[n]))
    # (candidates have no place in the order: without the bias)
    att_all = attention(seq.Documents([m], [n]), causal=False, buckets=None)
    att_one = attention(seq.Documents([1], [n]), causal=False, buckets=None)
    single = cand[:one_by_one]
    for layer in model.layers:
        q, k, v = layer.keys_values(obs)
        qc = layer.keys_values(cand)[0]
        cand = layer.rest(cand, seq.attend(att_all, qc, k, v)["out"])
        if one_by_one:
            qs = layer.keys_values(single)[0]
            single = layer.rest(single, torch.cat([seq.attend(att_one, qs[i:i + 1], k, v)["out"]
                                                   for i in range(one_by_one)]))
        obs = layer.rest(obs, seq.attend(att_obs, q, k, v, table=layer.table)["out"])
    logits = model.head(norm(cand))
    return (logits, model.head(norm(single))) if one_by_one else logits


@torch.no_grad()
def rotary_answer(model, x_obs, y_obs, candidates, one_by_one=0):
    """The same with rotary positions: observations stand one after the other and their keys and
    values go into a cache, a candidate stands behind the last of them."""
    n, m = x_obs.shape[0], candidates.shape[0]
    obs = model.embed(x_obs, y_obs, torch.ones(n, dtype=torch.bool, device="cuda"))
    cand = model.embed(candidates, torch.zeros(m, device="cuda"),
                       torch.zeros(m, dtype=torch.bool, device="cuda"))
    att_obs = attention(seq.Documents([n], prefix=[n]), buckets=None)
    att_all = attention(seq.Documents([m], [n]), causal=False, buckets=None)
    att_one = attention(seq.Documents([1], [n]), causal=False, buckets=None)
    place = torch.arange(n, dtype=torch.int32, device="cuda")
    behind = torch.full((m,), n, dtype=torch.int32, device="cuda")
    k, v = (torch.empty((n, KV_HEADS, HEAD), dtype=obs.dtype, device="cuda") for _ in range(2))
    o, c, s = ((x, torch.zeros_like(x)) for x in (obs, cand, cand[:one_by_one]))
    for layer in model.layers:
        y, x = layer.heads(*o)
        q, *new = y.split([HEADS, KV_HEADS, KV_HEADS], 1)
        turned = torch.empty((n, HEADS, HEAD), dtype=obs.dtype, device="cuda")
        layers.append_into(layer.rotary, place, place.long(), q, *new, turned, k, v)
        o = layer.rest(x, seq.attend(att_obs, turned, k, v)["out"])
        y, x = layer.heads(*c)
        c = layer.rest(x, seq.attend(att_all, layers.rotate(layer.rotary, behind, y[:, :HEADS]), k, v)["out"])
        if one_by_one:
            rows = []
            for i in range(one_by_one):
                y, x = layer.heads(s[0][i:i + 1], s[1][i:i + 1])
                q = layers.rotate(layer.rotary, behind[:1], y[:, :HEADS])
                rows.append(layer.rest(x, seq.attend(att_one, q, k, v)["out"]))
            s = tuple(torch.cat(x) for x in zip(*rows))
    logits = model.answers(*c)
    return (logits, model.answers(*s)) if one_by_one else logits


def expected_improvement(logits, best):
    """E[max(best - y, 0)] of the binned outcome."""
    centres = LOW + (torch.arange(BINS, device="cuda") + 0.5) * (HIGH - LOW) / BINS
    return torch.softmax(logits.float(), 1) @ (best - centres).clamp_min(0)


def main(steps=400, candidates=65536, log=print, order="bias"):
    torch.manual_seed(0)
    gen = torch.Generator().manual_seed(1)
    model = (RotarySurrogate if order == "rotary" else Surrogate)().cuda().bfloat16()
    losses = train(model, steps, gen, log=log)
    xs, ys, ((n, m),) = draw_runs(1, 64, 64, gen)
    cand = torch.rand((candidates, PARAMS), generator=gen).cuda()
    ask = rotary_answer if order == "rotary" else answer
    logits, single = ask(model, xs[:n], ys[:n], cand, one_by_one=4)
    ei = expected_improvement(logits, ys[:n].min())
    best = torch.topk(ei, 3)
    log(f"{candidates} candidates against {n} observations: best expected improvement "
        f"{[round(x, 4) for x in best.values.tolist()]} at {best.indices.tolist()}")
    bins = seq.logprob(logits[best.indices].contiguous(),
                       torch.full((3,), -1, dtype=torch.int64, device="cuda"), top=3)
    log(f"most likely outcome bins of these: {bins['top_id'].tolist()}")
    diff = (logits[:4].float() - single.float()).abs().max().item()
    log(f"one candidate at a time: logits within {diff:.3f} of the batch's")
    return {"losses": losses, "ei": ei, "diff": diff}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--order", choices=("bias", "rotary"), default="bias")
    args = ap.parse_args()
    main(args.steps, order=args.order)
