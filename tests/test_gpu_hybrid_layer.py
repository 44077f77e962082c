"""The hybrid pair of layers end to end: prefill, then decode, agrees with the longer
prefill, and its gradients with a difference of its output.

The pair is bfloat16 throughout (about twenty roundings of 2^-9 between input and output,
as random errors 1e-2; the KDN forward's own tolerance is 2e-2), so decode is held to
4e-2 of the output's norm.  The difference has bfloat16 noise of 1e-2 of the output's
norm, 1e-2 sqrt(N) |dout| / (2 e) = 0.02 sqrt(N) of a loss of N = B T D terms, against a
random direction's share |dx| |step| / sqrt(N) of about sqrt(N): 0.2 leaves room for the
truncation too."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_hybrid_pair():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import hybrid_layer
    finally:
        sys.path.pop(0)
    err, grad = hybrid_layer.main()
    assert err <= 4e-2
    assert grad <= 0.2
