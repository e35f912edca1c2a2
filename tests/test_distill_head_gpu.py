"""The head-fitting example end to end: forward, top logits, differentiable distillation,
the quantized head and sampling, on small sizes."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

pytestmark = pytest.mark.gpu


def test_head_is_fitted_and_deployed():
    import distill_head
    losses, deployed, labels, log_prob = distill_head.run(samples=2000, steps=40)
    assert losses[-1] < losses[0]
    # the int8 head is the float one to half a step of 127 per weight
    assert abs(deployed - losses[-1]) < 0.1 * losses[0]
    assert labels.shape == (2000,) and bool(((labels >= 0) & (labels < 10)).all())
    assert bool((log_prob <= 0).all()) and bool(torch.isfinite(log_prob).all())
