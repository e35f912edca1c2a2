"""Rows of class scores or logits at the ends of the operators' ranges: groups of equal
logits larger than a list holds, rows of millions of classes, scores past 2^24, long
lists, extreme temperatures, more rows than one launch takes.

Tolerances are those of test_logit_rows_gpu.py: sums of exponentials to REL = 1e-5 of
themselves and 2^-22 of the largest exponent, whatever the number of classes; what has no
rounding in it is compared exactly."""
import numpy as np
import pytest
import torch

import logit_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl
from test_logit_rows_gpu import (DEV, EPS, FLOATS, REL, TINY, TYPES, _check_distill,
                                 _check_sample, _check_top, _gumbel, _host, _logits, _norm,
                                 _rng, _teacher)

pytestmark = pytest.mark.gpu


# ------------------------------------------------- groups of equal logits

def _tied(rng, c, dtype):
    """Rows of 0, 1, 7 and 40 classes above a group of equal ones (in two rows another
    group below it), and a row of eleven values."""
    level = 30 if dtype == torch.int32 else 1.0
    x = torch.zeros((6, c), dtype=dtype)
    for r, above in enumerate((0, 1, 7, 40, 7)):
        x[r, rng.permutation(c)[:above]] = level
    x[3, rng.permutation(c)[:c // 3]] = -level
    x[4, rng.permutation(c)[:c // 2]] = -2 * level
    x[5] = torch.from_numpy(rng.integers(0, 11, c)).to(dtype)
    return x


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [90, 1000, 1025, 8000, 8193, 40001, 140000])
def test_sample_top_k_cuts_equal_logits_under_a_top_p(c, dtype):
    rng = _rng(20, c, TYPES.index(dtype))
    x = _tied(rng, c, dtype)
    noise = _gumbel(rng, x.shape[0], c)
    t = 30.0 if dtype == torch.int32 else 1.0
    for k in (50, 300, 2000):
        for p in (0.5, 0.95):
            got = bl.bitlogic_sample(x.to(DEV), noise.to(DEV), t, k, p)
            torch.cuda.synchronize()
            _check_sample(x, noise, t, k, p, 0.0, got)


@pytest.mark.parametrize("p", [1.0, 0.95])
def test_sample_top_k_above_the_rows_classes(p):
    """A row with fewer classes than the top-k asks for, more than a list holds, the last
    of them at the lowest score: all are kept."""
    rng = _rng(21)
    c = 140000
    x = torch.full((2, c), -2 ** 31, dtype=torch.int32)
    for r in range(2):
        at = rng.permutation(c)
        x[r, at[:5000]] = 0
        x[r, at[5000:60000]] = -2 ** 31 + 1
    noise = _gumbel(rng, 2, c)
    got = bl.bitlogic_sample(x.to(DEV), noise.to(DEV), 2.0 ** 30, 100000, p)
    torch.cuda.synchronize()
    _check_sample(x, noise, 2.0 ** 30, 100000, p, 0.0, got)
