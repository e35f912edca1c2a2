"""Dropout against the oracle: every element type, sizes on both sides of eight columns and of
a block's tasks, strides, alignments, offsets, gradients and graphs.  Which elements stay is
compared exactly; what stays is one product in 32 bits (2^-24 of itself) and one rounding to
its type."""
import numpy as np
import pytest
import torch

import draft_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}
FLOATS = [torch.float32, torch.float16, torch.bfloat16]
TYPES = [torch.int32] + FLOATS
SEED, OFFSET = 0x123456789ABCDEF0, 0xFEDCBA9876543210


def _x(rng, n, c, dtype):
    if dtype == torch.int32:
        return torch.from_numpy(rng.integers(-5, 65536, (n, c)).astype(np.int32))
    return torch.from_numpy(rng.normal(0, 3, (n, c)).astype(np.float32)).to(dtype)


def _check(y, x, p, seed=SEED, offset=OFFSET):
    want = oracle.dropout(x.detach().cpu().double().numpy(), p, seed, offset)
    assert y.dtype == (torch.float32 if x.dtype == torch.int32 else x.dtype)
    got = y.detach().cpu().double().numpy()
    assert np.array_equal(got == 0, want == 0)
    # a product and its factor rounded to 32 bits (2^-24 each), int32 counts below 2^24 exact
    off = (HALF_STEP[y.dtype] * (1 + 2.0 ** -20) + 2 * 2.0 ** -24) * np.abs(want)
    assert (np.abs(got - want) <= off + LEAST[y.dtype]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,c", [(1, 1), (3, 7), (5, 8), (33, 9), (64, 10), (70, 100), (9, 257),
                                 (2, 2047), (2, 2048), (3, 2049), (1, 6001)])
def test_sizes(n, c, dtype):
    rng = np.random.default_rng([11, n, c, TYPES.index(dtype)])
    x = _x(rng, n, c, dtype)
    for p in (0.0, 0.1, 0.5, 1.0):
        y = bl.bitlogic_dropout(x.to(DEV), p, SEED, OFFSET)
        torch.cuda.synchronize()
        _check(y, x, p)


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_in_place(dtype):
    rng = np.random.default_rng([12, TYPES.index(dtype)])
    wide = _x(rng, 12, 300, dtype)
    on = wide.to(DEV)
    for view in ((slice(None), slice(1, 100)), (slice(None, None, 3), slice(7, 263)),
                 (slice(2, 3), slice(5, 300))):
        _check(bl.bitlogic_dropout(on[view], 0.3, SEED, OFFSET), wide[view], 0.3)
    row = on[:1, 9:90].expand(6, -1)                      # one row read for all
    _check(bl.bitlogic_dropout(row, 0.3, SEED, OFFSET), wide[:1, 9:90].expand(6, -1), 0.3)
    out_type = torch.float32 if dtype == torch.int32 else dtype
    out = torch.full((12, 310), 5, dtype=out_type, device=DEV)
    assert bl.bitlogic_dropout(on[:, 1:300], 0.3, SEED, OFFSET,
                               out=out[:, 3:302]).data_ptr() == out[:, 3:].data_ptr()
    _check(out[:, 3:302], wide[:, 1:300], 0.3)
    assert (out[:, :3] == 5).all() and (out[:, 302:] == 5).all()
    if dtype != torch.int32:
        part = on[:, 3:202]
        bl.bitlogic_dropout(part, 0.3, SEED, OFFSET, out=part)
        _check(part, wide[:, 3:202], 0.3)
        assert torch.equal(on[:, 202:].cpu(), wide[:, 202:])
        with pytest.raises(bl.BitlogicError, match="overlaps"):
            bl.bitlogic_dropout(on[:, :9], 0.3, 1, out=on[:, 1:10])


def test_what_is_dropped_is_zero():
    x = torch.full((64, 40), np.inf, device=DEV)
    x[::2] = np.nan
    y = bl.bitlogic_dropout(x, 0.5, SEED, OFFSET)
    drop = torch.from_numpy(oracle.numbers(64, 40, SEED, OFFSET) < 32768)
    assert torch.equal(y.cpu() == 0, drop)
    assert torch.equal(torch.isnan(y.cpu()), ~drop & torch.isnan(x.cpu()))
    assert not bl.bitlogic_dropout(x, 1.0, SEED, OFFSET).any()


def test_offsets_and_refusals():
    rng = np.random.default_rng(13)
    x = _x(rng, 30, 70, torch.float32)
    on = x.to(DEV)
    for offset in (0, 1, 2 ** 32 - 1, 2 ** 32, 2 ** 63 - 1):
        _check(bl.bitlogic_dropout(on, 0.4, 3, offset), x, 0.4, 3, offset)
        at = torch.tensor([offset], dtype=torch.int64, device=DEV)
        _check(bl.bitlogic_dropout(on, 0.4, 3, at), x, 0.4, 3, offset)
    _check(bl.bitlogic_dropout(on, 0.4, 2 ** 64 - 1, 2 ** 64 - 1), x, 0.4, 2 ** 64 - 1,
           2 ** 64 - 1)
    assert bl.bitlogic_dropout(on[:0], 0.4, 3).shape == (0, 70)
    leaf = on[:0].clone().requires_grad_()
    bl.bitlogic_dropout(leaf, 0.4, 3).sum().backward()
    assert leaf.grad.shape == (0, 70)
    for seed, offset in ((-1, 0), (2 ** 64, 0), (0, -1), (0, 2 ** 64)):
        with pytest.raises(ValueError, match="seed and offset"):
            bl.bitlogic_dropout(on, 0.4, seed, offset)
    with pytest.raises(ValueError, match="2-D"):
        bl.bitlogic_dropout(on[0], 0.4, 1)
    with pytest.raises(ValueError, match="x's shape"):
        bl.bitlogic_dropout(on, 0.4, 1, out=torch.empty((30, 69), device=DEV))
    with pytest.raises(TypeError, match="offset has dtype"):
        bl.bitlogic_dropout(on, 0.4, 1, torch.zeros(1, device=DEV))


@pytest.mark.parametrize("dtype", FLOATS)
def test_gradient(dtype):
    rng = np.random.default_rng([14, FLOATS.index(dtype)])
    x, g = _x(rng, 37, 101, dtype), _x(rng, 37, 101, dtype)
    leaf = x.to(DEV).requires_grad_()
    y = bl.bitlogic_dropout(leaf, 0.3, SEED, OFFSET)
    grad, = torch.autograd.grad(y, leaf, g.to(DEV))
    _check(y, x, 0.3)
    _check(grad, g, 0.3)                                  # the same mask and factor
    if dtype == torch.float32:                            # it is linear: differences are exact
        step = 0.5 * torch.eye(101, device=DEV)[3]        # up to the roundings of both sides
        moved = bl.bitlogic_dropout(leaf.detach() + step, 0.3, SEED, OFFSET)
        slope = ((moved - y.detach()) / 0.5)[:, 3]
        ones = bl.bitlogic_dropout(torch.ones_like(leaf.detach()), 0.3, SEED, OFFSET)[:, 3]
        assert ((slope - ones).abs() <= 2.0 ** -21 * (2 * y.detach()[:, 3].abs() + 4)).all()
    # a gradient that is one number for all, and x with no need of one
    grad, = torch.autograd.grad(bl.bitlogic_dropout(leaf, 0.3, SEED, OFFSET).sum(), leaf)
    _check(grad, torch.ones((37, 101), dtype=dtype), 0.3)
    with torch.no_grad():
        assert not bl.bitlogic_dropout(leaf, 0.3, 1).requires_grad


def test_offset_raised_before_the_backward_pass_is_refused():
    leaf = torch.ones((4, 9), device=DEV, requires_grad=True)
    at = torch.tensor([5], dtype=torch.int64, device=DEV)
    y = bl.bitlogic_dropout(leaf, 0.3, SEED, at)
    at += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_streams_and_graph():
    rng = np.random.default_rng(15)
    x = _x(rng, 90, 333, torch.bfloat16)
    on = x.to(DEV)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    y = bl.bitlogic_dropout(on, 0.2, SEED, 4, stream=stream)
    stream.synchronize()
    _check(y, x, 0.2, offset=4)
    at = torch.tensor([8], dtype=torch.int64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = bl.bitlogic_dropout(on, 0.2, SEED, at)
        at += 1
    for turn in range(4):
        x = _x(rng, 90, 333, torch.bfloat16)
        on.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        _check(y, x, 0.2, offset=8 + turn)
        bl.bitlogic_dropout(on, 0.2, SEED, 77)


def test_rows_past_32_bit_offsets():
    """Elements past 2^32 bytes: the last rows of a tall tensor of one stride."""
    x = torch.ones((1, 1 << 16), dtype=torch.float16, device=DEV)
    out = bl.bitlogic_dropout(x.expand(40000, -1), 0.5, SEED, OFFSET)     # 5.2 GB
    drop = torch.from_numpy(oracle.numbers(1, 64, SEED, OFFSET) < 32768)
    assert torch.equal(out[:1, :64].cpu() == 0, drop)
    block, s, low = 65535 // 8, 39999, 0xFFFFFFFF
    c, k = [block, s, OFFSET & low, OFFSET >> 32], [SEED & low, SEED >> 32]
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [b >> 32 ^ c[1] ^ k[0], b & low, a >> 32 ^ c[3] ^ k[1], a & low]
        k = [k[0] + 0x9E3779B9 & low, k[1] + 0xBB67AE85 & low]
    keep = [h >= 32768 for w in c for h in (w & 0xFFFF, w >> 16)]
    assert (out[39999, -8:] != 0).cpu().tolist() == keep
    share = float((out[39000:] != 0).float().mean())
    assert abs(share - 0.5) < 6 * 0.5 / (1000 * 65536) ** 0.5


def test_forward_mode_is_refused():
    """A tangent is not dropped without a word: there is no forward-mode derivative."""
    x = torch.ones((4, 9), device=DEV)
    with torch.autograd.forward_ad.dual_level():
        for leaf in (x, x.clone().requires_grad_()):
            dual = torch.autograd.forward_ad.make_dual(leaf, torch.ones_like(x))
            with pytest.raises((RuntimeError, NotImplementedError)):
                bl.bitlogic_dropout(dual, 0.3, SEED)
            with torch.no_grad(), pytest.raises((RuntimeError, NotImplementedError)):
                bl.bitlogic_dropout(dual, 0.3, SEED)
        y = bl.bitlogic_dropout(x, 0.3, SEED)             # one without a tangent, beside it
        assert torch.equal(y, bl.bitlogic_dropout(x.clone(), 0.3, SEED))
    with pytest.raises((RuntimeError, NotImplementedError)):
        torch.func.jvp(lambda v: bl.bitlogic_dropout(v, 0.3, SEED), (x,), (x,))
