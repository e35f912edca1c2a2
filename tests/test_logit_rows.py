"""Argument checks of the calls on rows of class scores, which need no GPU, and the
64-bit oracle of their tests against values worked out by hand."""
import ctypes
import math

import numpy as np
import pytest
import torch

import logit_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl

FAKE = 0x10000                       # never dereferenced: every call fails before a launch
OK, ENULL, ESHAPE, EALIGN, EUNSUP, EHIP, EWS = range(7)
I32, F32, F16, BF16 = range(4)
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake-pointer argument checks run only where no GPU is visible")
    return bl.load_library()


def _top(lib, logits=FAKE, type=F32, rows=4, n=10, stride=10, k=3, t=1.0, values=FAKE,
         indices=FAKE, log_norm=FAKE):
    return lib.bitlogic_top_logits(logits, type, rows, n, stride, k, t, values, indices,
                                   log_norm, None)


def _distill(lib, logits=FAKE, type=F32, rows=4, n=10, stride=10, t=1.0, values=FAKE,
             top_type=F32, indices=FAKE, k=3, log_norm=None, tt=1.0, weight=None, loss=FAKE,
             grad=FAKE, grad_stride=10):
    return lib.bitlogic_distill(logits, type, rows, n, stride, t, values, top_type, indices, k,
                                log_norm, tt, weight, loss, grad, grad_stride, None)


def _sample(lib, logits=FAKE, type=F32, rows=4, n=10, stride=10, noise=FAKE, noise_stride=10,
            token=FAKE, log_prob=FAKE, sampling=True, t=1.0, k=0, p=1.0, m=0.0, **arrays):
    s = bl._Sampling(t, k, p, m)
    for name, value in arrays.items():
        setattr(s, name, value)
    return lib.bitlogic_sample(logits, type, rows, n, stride, noise, noise_stride,
                               ctypes.addressof(s) if sampling else None, token, log_prob, None)


@pytest.mark.parametrize("call", [_top, _distill, _sample])
def test_rows_are_checked(lib, call):
    for type in (-1, 4):
        assert call(lib, type=type) == EUNSUP
    assert call(lib, rows=-1) == ESHAPE
    assert call(lib, rows=1 << 31) == ESHAPE
    assert call(lib, n=0) == ESHAPE
    assert call(lib, n=(1 << 30) + 1) == ESHAPE
    assert call(lib, stride=-1) == ESHAPE
    assert call(lib, stride=(1 << 30) + 1) == ESHAPE
    assert call(lib, logits=None) == ENULL
    assert call(lib, logits=FAKE + 2) == EALIGN
    assert call(lib, type=BF16, logits=FAKE + 1) == EALIGN
    assert call(lib, rows=0) == OK and call(lib, rows=0, logits=None) == OK


def test_top_validation(lib):
    assert _top(lib, k=0) == ESHAPE
    assert _top(lib, k=1025) == EUNSUP
    for t in (0.0, -1.0, INF, NAN):
        assert _top(lib, t=t) == ESHAPE
    assert _top(lib, values=None) == ENULL and _top(lib, indices=None) == ENULL
    assert _top(lib, values=FAKE + 2) == EALIGN and _top(lib, indices=FAKE + 2) == EALIGN
    assert _top(lib, log_norm=FAKE + 2) == EALIGN


def test_distill_validation(lib):
    assert _distill(lib, k=0) == ESHAPE
    assert _distill(lib, k=1025) == EUNSUP
    for t in (0.0, -1.0, INF, NAN):
        assert _distill(lib, t=t) == ESHAPE and _distill(lib, tt=t) == ESHAPE
    assert _distill(lib, top_type=4) == EUNSUP
    assert _distill(lib, type=I32) == EUNSUP                      # scores have no gradient
    assert _distill(lib, grad_stride=9) == ESHAPE
    assert _distill(lib, grad_stride=(1 << 30) + 1) == ESHAPE
    assert _distill(lib, loss=None, grad=None) == ENULL
    assert _distill(lib, values=None) == ENULL and _distill(lib, indices=None) == ENULL
    for name in ("values", "indices", "log_norm", "weight", "loss", "grad"):
        assert _distill(lib, **{name: FAKE + 2}) == EALIGN, name


def test_sample_validation(lib):
    assert _sample(lib, sampling=False) == ENULL
    for t in (-1.0, INF, NAN):
        assert _sample(lib, t=t) == ESHAPE
    assert _sample(lib, k=-1) == ESHAPE
    for p in (-0.1, 1.1, NAN):
        assert _sample(lib, p=p) == ESHAPE and _sample(lib, m=p) == ESHAPE
    assert _sample(lib, noise=None) == ENULL and _sample(lib, token=None) == ENULL
    # arrays take the places of numbers that would be refused
    assert _sample(lib, t=NAN, k=-1, p=NAN, m=NAN, temperatures=FAKE, top_ks=FAKE, top_ps=FAKE,
                   min_ps=FAKE, rows=0) == OK
    assert _sample(lib, t=0.0, noise=None, temperatures=FAKE) == ENULL
    assert _sample(lib, noise_stride=-1) == ESHAPE
    for name in ("noise", "token", "log_prob", "temperatures", "top_ks", "top_ps", "min_ps"):
        assert _sample(lib, **{name: FAKE + 2}) == EALIGN, name


def test_binding_refuses_host_tensors_and_shapes():
    x = torch.zeros((2, 5))
    with pytest.raises(ValueError, match="on the GPU"):
        bl.bitlogic_top_logits(x, 2)
    with pytest.raises(ValueError, match="on the GPU"):
        bl.bitlogic_sample(x, x)
    with pytest.raises(TypeError, match="torch tensor"):
        bl.bitlogic_distill(x.numpy(), x, x)


# ------------------------------------------------------------ the oracle itself

def test_oracle_top():
    x = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0]])
    cls, norm = oracle.top(x, np.isinf(x), 5, 1.0)
    assert cls.tolist() == [[1, 2, 4, 0, -1]]
    assert abs(norm[0] - math.log(math.e + 2 * math.e ** 3 + math.e ** 2)) < 1e-12


def test_oracle_distill():
    # two classes at equal odds, a teacher sure of the first: log 2, gradient p - q
    loss, grad, *_ = oracle.distill(np.zeros(2), 1.0, np.array([4.0]), np.array([0]), 1.0)
    assert abs(loss - math.log(2)) < 1e-12 and np.allclose(grad, [-0.5, 0.5])
    # with the rest: q = (1/2, 1/2) against p = (1/3, 2/3)
    loss, grad, *_ = oracle.distill(np.zeros(3), 1.0, np.array([0.0]), np.array([1]), 1.0,
                                    math.log(2))
    want = 0.5 * math.log(0.5 * 3) + 0.5 * math.log(0.5 * 1.5)
    assert abs(loss - want) < 1e-12
    assert np.allclose(grad, [1 / 3 - 0.25, 1 / 3 - 0.5, 1 / 3 - 0.25])
    # an empty list has neither loss nor gradient
    loss, grad, *_ = oracle.distill(np.arange(3.0), 1.0, np.zeros(2), np.array([-1, 3]), 1.0)
    assert loss == 0 and (grad == 0).all()


def test_oracle_sample():
    x = np.log(np.array([0.1, 0.4, 0.4, 0.1])).astype(np.float32).astype(np.float64)
    none = np.zeros(4, bool)
    zero = np.zeros(4)
    kept = lambda *a: sorted(oracle.sample(x, none, zero, *a)[2])
    assert kept(1.0, 0, 1.0, 0.0) == [0, 1, 2, 3]
    assert kept(1.0, 1, 1.0, 0.0) == [1]
    assert kept(1.0, 3, 1.0, 0.0) == [0, 1, 2]
    assert kept(1.0, 0, 0.5, 0.0) == [1, 2]
    assert kept(1.0, 0, 0.3, 0.0) == [1]
    assert kept(1.0, 0, 0.0, 0.0) == [1]
    assert kept(1.0, 0, 1.0, 0.5) == [1, 2]
    assert oracle.sample(x, none, zero, 0.0, 0, 1.0, 0.0)[:2] == (1, 0.0)
    token, log_prob, _ = oracle.sample(x, none, np.array([9.0, 0, 0, 0]), 1.0, 0, 1.0, 0.0)
    assert token == 0 and abs(log_prob - math.log(0.1)) < 1e-6
    assert oracle.sample(x, ~none, zero, 1.0, 0, 1.0, 0.0)[0] == -1
