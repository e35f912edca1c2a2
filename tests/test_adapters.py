"""Argument checks of the adapter calls, which need no GPU, and their oracle against a worked
example."""
import ctypes

import numpy as np
import pytest
import torch

import adapter_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl

FAKE = 0x10000                       # never dereferenced: every call fails before a launch
FAR = FAKE + (1 << 24)
OK, ENULL, ESHAPE, EALIGN, EUNSUP, EHIP, EWS = range(7)
I32, F32, F16, BF16 = range(4)


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("fake-pointer argument checks run only where no GPU is visible")
    return bl.load_library()


def _set(**fields):
    s = bl._AdapterSet(FAKE, FAKE, F32, 3, 4, 10, 12, 1.0, None)
    for name, value in fields.items():
        setattr(s, name, value)
    return s


def _forward(lib, x=FAKE, x_type=F32, rows=5, stride=10, ids=FAKE, plan=FAKE, base=FAKE,
             base_type=F32, base_stride=12, out=FAR, out_stride=12, hidden=FAKE,
             workspace=FAKE, ws_bytes=1 << 40, set_=True, **fields):
    s = _set(**fields)
    return lib.bitlogic_adapters(x, x_type, rows, stride, ctypes.addressof(s) if set_ else None,
                                 ids, plan, base, base_type, base_stride, 1.0, out, out_stride,
                                 hidden, workspace, ws_bytes, None)


def _backward(lib, grad=FAKE, rows=5, grad_stride=12, x=FAKE, x_type=F32, stride=10, hidden=FAKE,
              ids=FAKE, plan=FAKE, grad_x=FAR, grad_x_stride=10, grad_down=FAR, grad_up=FAR,
              workspace=FAKE, ws_bytes=1 << 40, set_=True, **fields):
    s = _set(**fields)
    return lib.bitlogic_adapters_backward(grad, rows, grad_stride, x, x_type, stride, hidden,
                                          ctypes.addressof(s) if set_ else None, ids, plan,
                                          grad_x, grad_x_stride, grad_down, grad_up, workspace,
                                          ws_bytes, None)


@pytest.mark.parametrize("call", [_forward, _backward])
def test_sets_are_checked(lib, call):
    for bad in ({"weight_type": I32, "x_type": I32}, {"weight_type": 4}, {"x_type": F16},
                {"x_type": I32, "weight_type": BF16}, {"n_adapters": 4097}, {"rank": 129}):
        assert call(lib, **bad) == EUNSUP, bad
    for bad in ({"rows": -1}, {"rows": (1 << 27) + 1}, {"n_adapters": 0}, {"rank": 0},
                {"n_in": 0}, {"n_out": 0}, {"n_in": (1 << 24) + 1}, {"n_out": (1 << 24) + 1},
                {"stride": -1}, {"stride": (1 << 30) + 1}):
        assert call(lib, **bad) == ESHAPE, bad
    assert call(lib, set_=False) == ENULL
    for name in ("down", "up"):
        assert call(lib, **{name: None}) == ENULL, name
    for name in ("x", "down", "up", "scales", "hidden"):
        assert call(lib, **{name: FAKE + 2}) == EALIGN, name
    assert call(lib, plan=None, ids=None) == ENULL
    assert call(lib, plan=FAKE + 8) == EALIGN


def test_forward_validation(lib):
    assert _forward(lib, x=None) == ENULL and _forward(lib, out=None, hidden=None) == ENULL
    assert _forward(lib, base_type=BF16) == EUNSUP
    assert _forward(lib, base_type=I32, weight_type=F16, x_type=F16) == EUNSUP
    for bad in ({"base_stride": -1}, {"out_stride": 11}, {"out_stride": (1 << 30) + 1},
                {"rows": (1 << 20) + 1, "plan": None}):
        assert _forward(lib, **bad) == ESHAPE, bad
    for name in ("base", "out"):
        assert _forward(lib, **{name: FAKE + 2}) == EALIGN, name
    assert _forward(lib, plan=None, ids=FAKE + 2) == EALIGN
    # out is base, or apart from it and from x
    for bad in ({"out": FAKE + 40}, {"out": FAKE, "base": FAR},
                {"base": FAR, "out": FAR, "base_stride": 13}, {"base": FAR + 4},
                {"base": FAR, "base_type": I32}):
        assert _forward(lib, **bad) == ESHAPE, bad
    need = lib.bitlogic_adapters_workspace_bytes
    s = _set(n_in=5000)
    size = need(ctypes.addressof(s), 5, 1)
    assert size >= 5 * 4 * 4 and need(ctypes.addressof(s), (1 << 20) + 1, 0) == 0
    assert need(None, 5, 1) == 0 and need(ctypes.addressof(_set()), 5, 1) == 0
    wide = dict(n_in=5000, stride=5000, hidden=None)
    assert _forward(lib, **wide, ws_bytes=size - 1) == EWS
    assert _forward(lib, **wide, workspace=None) == EWS
    assert _forward(lib, **wide, workspace=FAKE + 8) == EALIGN
    assert _forward(lib, rows=0, x=None, out=None, hidden=None, plan=None, ids=None) == OK


def test_backward_validation(lib):
    for name in ("grad", "x", "hidden"):
        assert _backward(lib, **{name: None}) == ENULL, name
    assert _backward(lib, grad_x=None, grad_down=None, grad_up=None) == ENULL
    assert _backward(lib, plan=None) == ENULL                     # weights' gradients need one
    for bad in ({"grad_stride": -1}, {"grad_x_stride": 9},
                {"grad_x": None, "grad_down": None, "grad_up": None, "grad_stride": -1}):
        assert _backward(lib, **bad) == ESHAPE, bad
    for name in ("grad", "grad_x", "grad_down", "grad_up"):
        assert _backward(lib, **{name: FAR + 2}) == EALIGN, name
    s = _set()
    need = lib.bitlogic_adapters_backward_workspace_bytes(ctypes.addressof(s), 5)
    assert need >= 5 * 4 * 4
    assert _backward(lib, ws_bytes=need - 1) == EWS and _backward(lib, workspace=None) == EWS
    assert _backward(lib, workspace=FAKE + 8) == EALIGN
    assert lib.bitlogic_adapters_backward_workspace_bytes(None, 5) == 0
    assert _backward(lib, rows=1 << 27, n_in=1 << 24, stride=1 << 24, n_out=1 << 24,
                     grad_x_stride=1 << 24, rank=1, ws_bytes=1 << 62) == EUNSUP


def test_group_rows_validation(lib):
    bytes_, call = lib.bitlogic_group_rows_bytes, lib.bitlogic_group_rows
    need = bytes_(1000, 7)
    assert need >= 4000
    for bad in ((-1, 7), ((1 << 27) + 1, 7), (1000, 0), (1000, 4097)):
        assert bytes_(*bad) == 0
    assert call(FAKE, -1, 7, FAKE, need, None) == ESHAPE
    assert call(FAKE, 1000, 0, FAKE, need, None) == ESHAPE
    assert call(FAKE, 1000, 4097, FAKE, need, None) == EUNSUP
    assert call(None, 1000, 7, FAKE, need, None) == ENULL
    assert call(FAKE, 1000, 7, None, need, None) == ENULL
    assert call(FAKE + 2, 1000, 7, FAKE, need, None) == EALIGN
    assert call(FAKE, 1000, 7, FAKE + 8, need, None) == EALIGN
    assert call(FAKE, 1000, 7, FAKE, need - 1, None) == EWS
    assert call(None, 0, 7, None, 0, None) == OK


def test_binding_refuses():
    x, w = torch.zeros((2, 5)), torch.zeros((3, 4, 5))
    with pytest.raises(ValueError, match="on the GPU"):
        bl.bitlogic_adapters(x, w, w, None)
    with pytest.raises(ValueError, match="on the GPU"):
        bl.bitlogic_group_rows(torch.zeros(5, dtype=torch.int32), 3)
    with pytest.raises(ValueError, match="ids must be"):
        bl.bitlogic_group_rows(torch.zeros((5, 1), dtype=torch.int32), 3)


def test_oracle():
    x = np.array([[1.0, 2.0], [3.0, -1.0], [5.0, 5.0]])
    down, up = np.array([[[1.0, 1.0]], [[2.0, 0.0]]]), np.array([[[1.0], [0.5]], [[3.0], [-1.0]]])
    ids, scales = np.array([1, 0, 7]), np.array([2.0, 10.0])
    base = np.ones((3, 2))
    out, hidden, _ = oracle.forward(x, down, up, ids, scales, base, 0.5)
    assert hidden.tolist() == [[2.0], [2.0], [0.0]]
    assert out.tolist() == [[60.5, -19.5], [4.5, 2.5], [0.5, 0.5]]
    g = np.array([[1.0, 0.0], [0.0, 1.0], [9.0, 9.0]])
    (gx, _), (gd, _), (gu, _) = oracle.backward(g, x, down, up, ids, scales)
    assert gx.tolist() == [[60.0, 0.0], [1.0, 1.0], [0.0, 0.0]]
    assert gd.tolist() == [[[3.0, -1.0]], [[30.0, 60.0]]]
    assert gu.tolist() == [[[0.0], [4.0]], [[20.0], [0.0]]]
    order, starts = oracle.groups(np.array([1, -1, 0, 1, 2, 0]), 2)
    assert order.tolist() == [2, 5, 0, 3, 1, 4] and starts.tolist() == [0, 2, 4, 6]


def test_oracle_gradients_are_the_slopes():
    rng = np.random.default_rng(3)
    x, down, up = rng.normal(size=(6, 5)), rng.normal(size=(2, 3, 5)), rng.normal(size=(2, 4, 3))
    ids, scales, g = np.array([0, 1, 1, -1, 0, 1]), np.array([0.5, 2.0]), rng.normal(size=(6, 4))
    value = lambda: (oracle.forward(x, down, up, ids, scales, None, 1.0)[0] * g).sum()   # noqa: E731
    for leaf, (grad, _) in zip((x, down, up), oracle.backward(g, x, down, up, ids, scales)):
        for at in np.ndindex(leaf.shape):
            kept = leaf[at]
            leaf[at] = kept + 0.5                         # the value is linear in each
            high = value()
            leaf[at] = kept - 0.5
            low = value()
            leaf[at] = kept
            assert abs(high - low - grad[at]) < 1e-12 * (1 + abs(high) + abs(low))


def test_launches_past_2_32_lanes_are_refused(lib):
    """A row without a plan is a tile of its own: 2^20 of them by 256 blocks of columns."""
    wide = dict(rows=1 << 20, stride=10, n_out=1 << 18, base=None, out=1 << 45,
                out_stride=1 << 18)
    assert _forward(lib, plan=None, **wide) == EUNSUP
    assert b"one launch" in lib.bitlogic_last_error()


def _apart(**fields):
    """Buffers of five rows by 3 adapters 10 -> 12 of rank 4, none of which overlap."""
    names = ("x", "grad", "base", "out", "hidden", "grad_x", "grad_down", "grad_up", "down", "up",
             "ids", "plan", "scales", "workspace")
    out = {name: FAKE + (i << 20) for i, name in enumerate(names)}
    out.update(fields)
    return out


def _only(call, args):
    own = {"_forward": ("x", "base", "out", "hidden"),
           "_backward": ("x", "grad", "hidden", "grad_x", "grad_down", "grad_up")}[call.__name__]
    return {k: v for k, v in args.items()
            if k in own + ("down", "up", "ids", "plan", "scales", "workspace")
            or k not in _apart()}


def test_hidden_apart_from_what_is_read_and_written(lib):
    at = _apart()
    sizes = {"x": 200, "base": 240, "out": 240, "down": 480, "up": 576}
    for name, size in sizes.items():
        for hidden in (at[name], at[name] + size - 4, at[name] - 76):
            assert _forward(lib, **_only(_forward, _apart(hidden=hidden))) == ESHAPE, name
            assert b"hidden overlaps" in lib.bitlogic_last_error()
        for hidden in (at[name] + size, at[name] - 80):
            assert _forward(lib, **_only(_forward, _apart(hidden=hidden))) == EHIP, name
    # a base that is not there, an output that is not there
    assert _forward(lib, **_only(_forward, _apart(base=None, hidden=at["base"]))) == EHIP
    assert _forward(lib, **_only(_forward, _apart(out=None, hidden=at["out"]))) == EHIP
    assert _forward(lib, **_only(_forward, _apart(out=None, hidden=at["up"]))) == EHIP
    assert _forward(lib, **_only(_forward, _apart(ids=at["hidden"], plan=None))) == ESHAPE
    assert _forward(lib, **_only(_forward, _apart(scales=at["hidden"] + 16))) == ESHAPE


def test_gradients_apart_from_what_is_read_and_written(lib):
    at = _apart()
    sizes = {"x": 200, "grad": 240, "hidden": 80, "grad_x": 200, "grad_down": 480,
             "grad_up": 576, "down": 480, "up": 576}
    for out in ("grad_x", "grad_down", "grad_up"):
        for name, size in sizes.items():
            if name == out:
                continue
            for where in (at[name], at[name] + size - 4, at[name] - sizes[out] + 4):
                assert _backward(lib, **_only(_backward, _apart(**{out: where}))) == ESHAPE
                assert b"overlaps" in lib.bitlogic_last_error()
            for where in (at[name] + size, at[name] - sizes[out]):
                assert _backward(lib, **_only(_backward, _apart(**{out: where}))) == EHIP
        assert _backward(lib, **_only(_backward, _apart(**{out: at["scales"]}))) == ESHAPE
    # what is not read: x and hidden beside the gradient of x alone
    for name in ("x", "hidden"):
        assert _backward(lib, **_only(_backward, _apart(
            grad_x=at[name], grad_down=None, grad_up=None))) == EHIP
    assert _backward(lib, **_only(_backward, _apart(
        grad_up=at["up"], grad_x=None, grad_down=None))) == EHIP
    # rows between each other's: 10 columns of x's gradient beside 12 of out's
    wide = dict(grad_stride=30, grad_x_stride=30)
    for where, want in ((12, EHIP), (20, EHIP), (11, ESHAPE), (21, ESHAPE)):
        args = _apart(grad_x=at["grad"] + 4 * where, **wide)
        assert _backward(lib, **_only(_backward, args)) == want, where
    args = _apart(grad_x=at["grad"] - 4 * 10, **wide)
    assert _backward(lib, **_only(_backward, args)) == EHIP
    args = _apart(grad_x=at["grad"] + 4 * 12, grad_stride=30, grad_x_stride=31)
    assert _backward(lib, **_only(_backward, args)) == ESHAPE
