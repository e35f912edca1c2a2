"""Argument checks of draft verification and dropout, which need no GPU, and their 64-bit
oracles against values worked out by hand and published ones."""
import ctypes
import math

import numpy as np
import pytest
import torch

import draft_oracle as oracle
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


def _verify(lib, logits=FAKE, type=F32, requests=4, n=10, stride=10, request_stride=40,
            noise=FAKE, noise_stride=10, accepted=FAKE, token=FAKE, log_prob=FAKE,
            workspace=FAKE, ws_bytes=1 << 40, drafts=True, **fields):
    d = bl._Drafts(FAKE, None, FAKE, F32, 3, 10, 30, FAKE, 1.0, 1.0, None, None)
    for name, value in fields.items():
        setattr(d, name, value)
    return lib.bitlogic_verify(logits, type, requests, n, stride, request_stride,
                               ctypes.addressof(d) if drafts else None, noise, noise_stride,
                               accepted, token, log_prob, workspace, ws_bytes, None)


def _dropout(lib, x=FAKE, type=F32, rows=4, n=10, stride=10, p=0.5, seed=1, offset=2, at=None,
             out=FAKE + (1 << 20), out_stride=10):
    return lib.bitlogic_dropout(x, type, rows, n, stride, p, seed, offset, at, out, out_stride,
                                None)


def test_verify_validation(lib):
    for type in (-1, 4):
        assert _verify(lib, type=type) == EUNSUP and _verify(lib, draft_type=type) == EUNSUP
    for bad in ({"requests": -1}, {"requests": 1 << 29}, {"n": 0}, {"n": (1 << 30) + 1},
                {"stride": -1}, {"stride": (1 << 30) + 1}, {"request_stride": -1},
                {"request_stride": (1 << 40) + 1}, {"draft_row_stride": -1},
                {"draft_request_stride": -1}, {"draft_request_stride": (1 << 40) + 1},
                {"n_drafted": -1}, {"n_drafted": 2 ** 31 - 1}, {"noise_stride": -1}):
        assert _verify(lib, **bad) == ESHAPE, bad
    for t in (-1.0, INF, NAN):
        assert _verify(lib, temperature=t) == ESHAPE
        assert _verify(lib, draft_temperature=t) == ESHAPE
        assert _verify(lib, temperature=t, temperatures=FAKE, draft_temperature=t,
                       draft_temperatures=FAKE, requests=0) == OK
    assert _verify(lib, drafts=False) == ENULL
    for name in ("logits", "noise", "accepted", "token", "drafted", "uniform"):
        assert _verify(lib, **{name: None}) == ENULL, name
    assert _verify(lib, temperature=0.0, temperatures=FAKE, noise=None) == ENULL
    for name in ("logits", "draft_logits", "noise", "accepted", "token", "log_prob", "drafted",
                 "uniform", "lengths", "temperatures", "draft_temperatures"):
        assert _verify(lib, **{name: FAKE + 2}) == EALIGN, name
    assert _verify(lib, requests=0, logits=None) == OK


def test_verify_workspace(lib):
    need = lib.bitlogic_verify_workspace_bytes
    assert need(100, 5, 100) == 0 and need(0, 5, 50000) == 0
    for bad in ((-1, 5, 50000), (5, -1, 50000), (1 << 29, 3, 50000), (5, 5, 0)):
        assert need(*bad) == 0
    for requests, drafts, n in ((1, 0, 50000), (1, 4, 131072), (300, 5, 50000)):
        size = need(requests, drafts, n)
        assert size >= requests * (drafts + 1) * 32
        args = dict(requests=requests, n_drafted=drafts, n=n, stride=n, noise_stride=n,
                    draft_row_stride=n)
        assert _verify(lib, **args, ws_bytes=size - 1) == EWS
        assert _verify(lib, **args, workspace=None, ws_bytes=0) == EWS
        assert _verify(lib, **args, workspace=FAKE + 4) == EALIGN


def test_dropout_validation(lib):
    for type in (-1, 4):
        assert _dropout(lib, type=type) == EUNSUP
    for bad in ({"rows": -1}, {"rows": 1 << 31}, {"n": 0}, {"n": (1 << 30) + 1}, {"stride": -1},
                {"stride": (1 << 30) + 1}, {"out_stride": 9}, {"out_stride": (1 << 30) + 1},
                {"p": -0.01}, {"p": 1.01}, {"p": NAN}):
        assert _dropout(lib, **bad) == ESHAPE, bad
    assert _dropout(lib, x=None) == ENULL and _dropout(lib, out=None) == ENULL
    assert _dropout(lib, x=FAKE + 2) == EALIGN and _dropout(lib, out=FAKE + 2) == EALIGN
    assert _dropout(lib, at=FAKE + 4) == EALIGN
    assert _dropout(lib, type=BF16, x=FAKE + 1) == EALIGN
    # out is x or apart from it
    for bad in ({"out": FAKE + 4}, {"out": FAKE, "out_stride": 11}, {"out": FAKE + 39 * 4},
                {"x": FAKE + 8, "out": FAKE}):
        assert _dropout(lib, **bad) == ESHAPE, bad
    assert _dropout(lib, rows=0, x=None, out=None) == OK


def test_binding_refuses():
    x = torch.zeros((2, 3, 5))
    with pytest.raises(ValueError, match="on the GPU"):
        bl.bitlogic_verify(x, x, x, x, x)
    with pytest.raises(TypeError, match="torch tensor"):
        bl.bitlogic_verify(x.numpy(), x, x, x, x)
    with pytest.raises(ValueError, match="on the GPU"):
        bl.bitlogic_dropout(x[0], 0.5, 1)


# ------------------------------------------------------------ the oracles

def test_generator_gives_published_numbers():
    """The known answer of Philox 4x32 with ten rounds at counter and key zero."""
    def words(h):
        return [int(h[2 * i]) | int(h[2 * i + 1]) << 16 for i in range(4)]
    assert words(oracle.numbers(1, 8, 0, 0)[0]) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c,
                                                    0x9b00dbd8]


def test_dropout_oracle():
    x = np.ones((40, 50))
    y = oracle.dropout(x, 0.25, 7, 9)
    assert set(np.unique(y)) == {0.0, 4 / 3}
    assert abs((y == 0).mean() - 0.25) < 0.05          # 2000 draws: five deviations are 0.048
    assert np.array_equal(oracle.dropout(x, 0.0, 7, 9), x)
    assert not oracle.dropout(x, 1.0, 7, 9).any()
    assert not np.array_equal(y, oracle.dropout(x, 0.25, 7, 10))
    assert not np.array_equal(y, oracle.dropout(x, 0.25, 8, 9))


def _one(p, q, drafted, u, noise, t=1.0, tq=1.0):
    with np.errstate(divide="ignore"):
        x = np.log(np.array(p, float))
        y = None if q is None else np.log(np.array(q, float))
    return oracle.verify(x, np.isinf(x), np.array(drafted), y, None if q is None else np.isinf(y),
                         np.array(u), np.array(noise, float), t, tq)


def test_verify_oracle():
    p = [[0.5, 0.5, 0.0], [0.1, 0.2, 0.7]]
    q = [[0.25, 0.25, 0.5]]
    zero = [0.0, 0.0, 0.0]
    assert _one(p, q, [0], [0.99], zero)[:2] == (1, 2)            # p / q = 2: always stands
    assert _one(p, q, [2], [0.0], zero)[:2] == (0, 0)             # p = 0: never
    assert _one(p, q, [2], [0.5], [0.0, 0.1, 0.0])[:2] == (0, 1)  # drawn from (1, 1, 0) / 2
    assert _one(p[::-1], [[0.2, 0.1, 0.7]], [0], [0.49], zero)[0] == 1
    assert _one(p[::-1], [[0.2, 0.1, 0.7]], [0], [0.51], [9, 0, 9])[:2] == (0, 1)   # only p > q
    assert _one(p, None, [0], [0.49], zero)[0] == 1               # q is one at the draft
    assert _one(p, None, [0], [0.51], [9, 0, 9])[:2] == (0, 1)    # the draft itself is out
    assert _one(p, None, [], [], [0, 1, 2])[:2] == (0, 1)
    assert _one(p, None, [-1], [0.0], [0, 1, 2])[:2] == (0, 1)
    assert _one(p, q, [0], [0.9], zero, t=0.0)[:2] == (1, 2)      # greedy: first of equals
    assert _one(p, q, [1], [0.0], zero, t=0.0) == (0, 0, 0.0)
    assert _one([[0, 0, 0]], None, [], [], zero) == (0, -1, -np.inf)
    assert abs(_one(p, q, [0], [0.99], zero)[2] - np.log(0.7)) < 1e-15
