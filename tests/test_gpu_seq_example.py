"""The example that runs the sequence operators together: it learns, and its batch and
single-row answers agree."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_in_context_surrogate():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import in_context_surrogate as ex
    finally:
        sys.path.pop(0)
    lines = []
    r = ex.main(steps=200, candidates=4099, log=lines.append)
    print("\n".join(lines), flush=True)
    last = sum(r["losses"][-10:]) / 10
    # a model that knows only the outcomes' overall distribution, a standard normal one in
    # bins of 1/16, cannot get below its entropy, log(16 sqrt(2 pi e)) = 4.19: below that it
    # has learned to read the observations
    assert last < 4.19 - 0.3, last
    assert r["ei"].isfinite().all() and (r["ei"] >= 0).all()
    # the same sums in other orders, rounded to 8 bits some dozen times on the way
    assert r["diff"] < 0.5
