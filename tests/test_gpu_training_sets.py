"""Tensor sets and handles of the training-step operators on the GPU where their life is not the simplest one: several host threads,
side streams, an Ops that goes before its sets, parameters of mixed kinds, long chunks.

Tolerances (u = 2^-24) are those of test_gpu_training.py: norm 12 u, m 4 u and v 5 u of the magnitudes of their terms, p 3 u |p| + u |p1| +
24 u of the update with those magnitudes in m's place.
"""
import os
import subprocess
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    import torch
    from paper_2609_23898_b200 import training
    assert torch.cuda.is_available()
    o = training.Ops()
    yield o
    o.status()


def test_a_set_used_at_once_on_a_side_stream(ops):
    """A non-blocking stream does not wait for the copies that made the set (2.6 MB of records here)."""
    import torch
    from paper_2609_23898_b200 import training as R
    flat = torch.full((20000 * 100,), 2.0, device="cuda")
    grads = list(flat.split(100))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(5):
            o = R.Ops()
            s = R.TensorSet(o, grads=grads)
            out = s.grad_norm(1.0)
            o.status()
            n64 = 2 * np.sqrt(flat.numel())
            assert abs(out[0].item() - n64) <= 12 * U * n64
