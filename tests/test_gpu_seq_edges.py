"""The sequence operators at their edges, on the GPU against the fp64 oracle: what lies outside
the documents, extremes of caps, offsets and probabilities, and calls of unusual sizes. Cases
and bounds are those of test_gpu_seq.py; what goes beyond them stands at each test."""
import math

import numpy as np
import pytest

from test_gpu_seq import TYPES, Case, _torch_dtype, near  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _announce(request):
    print(f"\n[gpu] {request.node.nodeid}", flush=True)
    yield


# ------------------------------------------------------------------ caps without a bias
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv", [(96, 2), (24, 3), (2, 2)])   # one and two groups, few rows
@pytest.mark.parametrize("cap,bias", [(30.0, "none"), (30.0, "one"), (5.0, "slope"), (0.0, "none")])
def test_attend_whole_tiles(dtype, dim, heads, kv, cap, bias):
    """Tiles that every row sees, whose scores are not touched between the cap and the maximum."""
    for causal in (False, True):
        for grad in (False, True):
            Case(dtype, [(330, 330), (130, 400)], heads, kv, dim, causal=causal, cap=cap, bias=bias,
                 size=3.0, grad=grad).check()


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_scores_that_grow(dtype):
    """Every tile's scores are far above those before it, by more than the type's range: the
    running maximum has to follow."""
    import torch
    for heads, kv in ((96, 2), (24, 3), (2, 2)):
        for cap in (0.0, 60.0):
            c = Case(dtype, [(200, 500)], heads, kv, 64, causal=False, cap=cap)
            c.q[:] = 1.0
            c.k[:] = torch.randn((500, kv, 64), generator=torch.Generator().manual_seed(1)).cuda().to(c.dt)
            c.k[:, :, :8] += (torch.arange(500, device="cuda") // 16).to(c.dt)[:, None, None]
            c.check()
