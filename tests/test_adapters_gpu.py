"""Low-rank adapters against the 64-bit oracle: every type, ranks and widths on both sides of
each kernel's limits, rows by plan and by themselves, rows without an adapter, strides,
gradients, streams and graphs; rows by group against a stable sort.

Tolerances.  A sum of k products in 32 bits is within 2 k 2^-24 of the sum of their absolute
values, whatever the order (2: the matrix cores may cut where others round).  In 16-bit types
down x enters the second product as two bfloat16, 2^-16 of itself.  `sizes` are the sums of
absolute values through both products.  Results are rounded to their type once."""
import numpy as np
import pytest
import torch

import adapter_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
F32, F16, BF16, I32 = torch.float32, torch.float16, torch.bfloat16, torch.int32
TYPES = [F32, F16, BF16, I32]                             # of x; int32 beside float32 adapters
HALF_STEP = {F32: 2.0 ** -24, F16: 2.0 ** -11, BF16: 2.0 ** -8}
LEAST = {F32: 1e-37, F16: 2.0 ** -24, BF16: 1e-37}


def _rng(*key):
    return np.random.default_rng([17, *[int(k) for k in key]])


def _normal(rng, shape, dtype, spread=1.0):
    return torch.from_numpy(rng.normal(0, spread, shape).astype(np.float32)).to(dtype)


def _np(t):
    return t.detach().cpu().double().numpy()


def _close(got, want, sizes, terms, name=""):
    dtype = got.dtype
    off = sizes * (2 * terms * 2.0 ** -24 + (0 if dtype == F32 else 2.0 ** -16))
    off = off + HALF_STEP[dtype] * (np.abs(want) + off) + LEAST[dtype]
    got = _np(got)
    assert got.shape == want.shape
    # (rounding takes what is past the type's largest value to an infinity of its sign)
    most = torch.finfo(dtype).max
    past = (np.abs(want) + off > most) & np.isinf(got) & (np.sign(got) == np.sign(want))
    with np.errstate(invalid="ignore"):
        bad = ~(np.abs(got - want) <= off) & ~past
    assert not bad.any(), (name, np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])


class Case:
    def __init__(self, key, n, f, c, r, g, type_, none=0.1, order="mixed", base=True):
        rng = _rng(*key, n, f, c, r, g, TYPES.index(type_))
        self.dtype = F32 if type_ == I32 else type_
        if type_ == I32:
            self.x = torch.from_numpy(rng.integers(0, 641, (n, f)).astype(np.int32))
            self.base = torch.from_numpy(rng.integers(-10 ** 6, 10 ** 6, (n, c)).astype(np.int32))
            self.base_scale = 1 / 128
        else:
            self.x, self.base = _normal(rng, (n, f), type_), _normal(rng, (n, c), type_)
            self.base_scale = 1.0 if n % 2 else 0.75
        if not base:
            self.base = None
        self.down = _normal(rng, (g, r, f), self.dtype, f ** -0.5)
        self.up = _normal(rng, (g, c, r), self.dtype, 0.5)
        ids = rng.integers(0, g, n)
        ids[rng.random(n) < none] = rng.choice([-1, g, 2 ** 31 - 1, -2 ** 31])
        self.ids = torch.from_numpy((np.sort(ids) if order == "runs" else ids).astype(np.int32))
        self.scales = torch.from_numpy(rng.uniform(0.5, 2, g).astype(np.float32))
        self.grad = _normal(rng, (n, c), self.dtype)
        self.n, self.f, self.c, self.r, self.g = n, f, c, r, g

    def on(self):
        move = lambda v: None if v is None else v.to(DEV)                        # noqa: E731
        return [move(v) for v in (self.x, self.down, self.up, self.ids, self.scales, self.base)]

    def host(self):
        return [_np(v) for v in (self.x, self.down, self.up)]

    def want(self):
        x, down, up = self.host()
        return oracle.forward(x, down, up, self.ids.numpy(), _np(self.scales),
                              None if self.base is None else _np(self.base),
                              float(np.float32(self.base_scale)))

    def check(self, out, hidden=None):
        want, h, sizes = self.want()
        # the term of the base and its sum with the other
        _close(out, want, sizes, self.f + self.r + 8, "out")
        if hidden is not None:
            x, down, _ = self.host()
            each = np.zeros(h.shape)
            for s, a in enumerate(self.ids.numpy()):
                if 0 <= a < self.g:
                    each[s] = np.abs(down[a]) @ np.abs(x[s])
            _close(hidden, h, each, self.f + 8, "hidden")

    def check_grads(self, gx, gd, gu):
        x, down, up = self.host()
        want = oracle.backward(_np(self.grad), x, down, up, self.ids.numpy(), _np(self.scales))
        for got, (grad, sizes), terms, name in zip(
                (gx, gd, gu), want, (self.c + self.r, self.c + self.n, self.f + self.n),
                ("grad_x", "grad_down", "grad_up")):
            if got is not None:
                _close(got, grad, sizes, terms + 8, name)

    def run(self, **kw):
        x, down, up, ids, scales, base = self.on()
        got = bl.bitlogic_adapters(x, down, up, ids, scales, base, self.base_scale,
                                   want_hidden=True, **kw)
        torch.cuda.synchronize()
        return got

    def backward(self, hidden, plan=None, **kw):
        x, down, up, ids, scales, _ = self.on()
        kw.setdefault("want_x", self.x.dtype != I32)
        got = bl.bitlogic_adapters_backward(self.grad.to(DEV), x, hidden, down, up, ids, scales,
                                            plan, **kw)
        torch.cuda.synchronize()
        return got

    def check_all(self):
        out, hidden = self.run()
        self.check(out, hidden)
        self.check_grads(*self.backward(hidden))


SHAPES = [  # rows, n_in, n_out, rank, adapters
    (1, 1, 1, 1, 1), (1, 100, 100, 8, 3), (5, 7, 3, 2, 2), (16, 10, 10, 4, 16),
    (17, 33, 65, 16, 2), (40, 100, 100, 8, 5), (70, 129, 31, 3, 1), (33, 64, 32, 17, 7),
    (100, 255, 257, 24, 3), (65, 512, 100, 32, 4), (64, 100, 513, 33, 2), (90, 520, 530, 5, 90),
    (31, 1030, 77, 64, 2), (45, 65, 2051, 65, 3), (50, 1500, 1027, 128, 2), (3, 4100, 2000, 16, 2),
    (200, 600, 40, 100, 3)]


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_shapes(shape, type_):
    Case((1,), *shape, type_).check_all()


@pytest.mark.parametrize("type_", TYPES)
@pytest.mark.parametrize("n,none", [(1, 1.0), (12, 0.5), (16, 0.0), (300, 0.95), (40, 1.0)])
def test_rows_without_an_adapter(n, none, type_):
    case = Case((2,), n, 90, 70, 6, 4, type_, none=none)
    case.check_all()
    case = Case((2,), n, 700, 600, 6, 4, type_, none=none, base=False)
    case.check_all()


@pytest.mark.parametrize("n", [3000, 9000])
@pytest.mark.parametrize("order", ["mixed", "runs"])
@pytest.mark.parametrize("type_", TYPES)
def test_many_rows(n, order, type_):
    """Groups of several chunks, whose parts of the gradients are joined."""
    Case((3,), n, 100, 90, 9, 3, type_, order=order).check_all()
    Case((3,), n, 20, 600, 20, 2, type_, order=order).check_all()


def test_few_rows_are_the_same_by_themselves_and_by_plan():
    for type_ in TYPES:
        case = Case((4,), 13, 700, 650, 20, 3, type_)
        alone, h1 = case.run()
        plan = bl.bitlogic_group_rows(case.ids.to(DEV), 3)
        grouped, h2 = case.run(plan=plan)
        case.check(alone, h1)
        case.check(grouped, h2)
        x, down, up, _, scales, base = case.on()
        again, _ = bl.bitlogic_adapters(x, down, up, None, scales, base, case.base_scale, plan)
        assert torch.equal(again, grouped)
        gx = case.backward(None, want_down=False, want_up=False, want_x=True)[0] \
            if type_ != I32 else None
        case.check_grads(gx, *case.backward(h2, plan)[1:])


def test_a_row_does_not_depend_on_others():
    """Infinities and NaNs stay in their rows and, among gradients, in their adapters."""
    for type_ in (F32, F16, BF16):
        case = Case((5,), 60, 300, 280, 12, 3, type_, none=0.1)
        x, down, up, ids, scales, base = case.on()
        clean, h = bl.bitlogic_adapters(x, down, up, ids, scales, base, case.base_scale,
                                        want_hidden=True)
        clean_grads = bl.bitlogic_adapters_backward(case.grad.to(DEV), x, h, down, up, ids,
                                                    scales)
        bad = [int((ids == 1).nonzero()[0]), int((ids == 1).nonzero()[-1])]
        x[bad[0]], x[bad[1], 5] = float("nan"), float("inf")
        base[(ids < 0) | (ids > 2)] = float("-inf")
        out, h = bl.bitlogic_adapters(x, down, up, ids, scales, base, case.base_scale,
                                      want_hidden=True)
        keep = torch.ones(60, dtype=torch.bool, device=DEV)
        keep[bad] = False
        adapted = (ids >= 0) & (ids <= 2)
        assert torch.equal(out[keep & adapted], clean[keep & adapted])
        assert (out[~adapted] == float("-inf")).all()
        assert torch.isnan(out[bad[0]]).all() and not torch.isfinite(out[bad[1]]).any()
        grads = bl.bitlogic_adapters_backward(case.grad.to(DEV), x, h, down, up, ids, scales)
        assert torch.equal(grads[0], clean_grads[0])      # (linear: x is not in it)
        for g, c in zip(grads[1:], clean_grads[1:]):
            assert torch.equal(g[[0, 2]], c[[0, 2]]) and torch.isnan(g[1]).any()


def test_large_values_of_float16():
    """down x past float16's range, with a result within it."""
    case = Case((6,), 40, 200, 100, 8, 2, F16)
    case.x = (case.x * 4000).to(F16)
    case.down = (case.down * 100).to(F16)
    case.up = (case.up / 4000).to(F16)
    out, hidden = case.run()
    assert hidden.abs().max() > 3e5
    case.check(out, hidden)
    case.check_grads(*case.backward(hidden))


def test_strides_outputs_and_in_place():
    for type_ in TYPES:
        for f, c in ((37, 45), (700, 650)):
            case = Case((7,), 50, f, c, 7, 3, type_)
            x, down, up, ids, scales, base = case.on()
            wide = torch.zeros((50, f + 9), dtype=x.dtype, device=DEV)
            wide[:, 5:f + 5] = x
            wide_base = torch.zeros((50, c + 3), dtype=base.dtype, device=DEV)
            wide_base[:, 1:c + 1] = base
            wide_out = torch.full((50, c + 4), 7.0, dtype=case.dtype, device=DEV)
            hidden = torch.empty((50, 7), device=DEV)
            out, h = bl.bitlogic_adapters(
                wide[:, 5:f + 5], down, up, ids, scales, wide_base[:, 1:c + 1], case.base_scale,
                out=wide_out[:, 3:c + 3], hidden=hidden)
            assert h is hidden
            case.check(out, hidden)
            assert (wide_out[:, :3] == 7).all() and (wide_out[:, c + 3:] == 7).all()
            if type_ != I32:
                into = wide_base[:, 1:c + 1]
                got, _ = bl.bitlogic_adapters(x, down, up, ids, scales, into, case.base_scale,
                                              out=into)
                assert torch.equal(got, out)
                assert (wide_base[:, 0] == 0).all() and (wide_base[:, c + 1:] == 0).all()
                wide_g = torch.zeros((50, c + 1), dtype=case.dtype, device=DEV)
                wide_g[:, 1:] = case.grad.to(DEV)
                wide_gx = torch.full((50, f + 2), 7.0, dtype=case.dtype, device=DEV)
                grads = bl.bitlogic_adapters_backward(
                    wide_g[:, 1:], wide[:, 5:f + 5], hidden, down, up, ids, scales,
                    grad_x=wide_gx[:, 1:f + 1])
                case.check_grads(*grads)
                assert (wide_gx[:, 0] == 7).all() and (wide_gx[:, f + 1] == 7).all()
            # one row of x and base for all
            case.x, case.base = case.x[:1].expand(50, f), case.base[:1].expand(50, c)
            out, _ = bl.bitlogic_adapters(x[:1].expand(50, f), down, up, ids, scales,
                                          base[:1].expand(50, c), case.base_scale)
            case.check(out)


def test_one_scale_for_all():
    case = Case((8,), 60, 80, 70, 5, 4, F32)
    case.scales[:] = 1.25
    x, down, up, ids, _, base = case.on()
    out, h = bl.bitlogic_adapters(x, down, up, ids, 1.25, base, case.base_scale, want_hidden=True)
    case.check(out, h)
    case.check_grads(*bl.bitlogic_adapters_backward(case.grad.to(DEV), x, h, down, up, ids, 1.25))


@pytest.mark.parametrize("type_", TYPES)
def test_autograd(type_):
    for n in (9, 200):
        case = Case((9,), n, 60, 50, 6, 3, type_)
        x, down, up, ids, scales, base = case.on()
        leaves = [v.requires_grad_() for v in ([] if type_ == I32 else [x])
                  + [down, up] + ([] if type_ == I32 else [base])]
        out = bl.bitlogic_adapt(x, down, up, ids, scales, base, case.base_scale)
        case.check(out)
        grads = list(torch.autograd.grad(out, leaves, case.grad.to(DEV)))
        gx = grads.pop(0) if type_ != I32 else None
        case.check_grads(gx, *grads[:2])
        if type_ != I32:
            want = _np(case.grad) * case.base_scale
            _close(grads[2], want, np.abs(want), 1)
        # the weights of one side alone, and a gradient that is one number for all
        case.grad = torch.ones_like(case.grad)
        out = bl.bitlogic_adapt(x.detach(), down.detach(), up, ids, scales, None)
        case.check_grads(None, None, torch.autograd.grad(out.sum(), up)[0])
        out = bl.bitlogic_adapt(x.detach(), down, up.detach(), ids, scales, None)
        case.check_grads(None, torch.autograd.grad(out.sum(), down)[0], None)


def test_gradients_are_the_slopes():
    """Differences of the sum of out * grad, which is linear in every element of x, down and
    up: exact but for the roundings of two float32 outputs."""
    case = Case((10,), 24, 20, 18, 3, 2, F32)
    x, down, up, ids, scales, base = case.on()
    g = case.grad.to(DEV).double()
    leaves = [v.requires_grad_() for v in (x, down, up)]
    out = bl.bitlogic_adapt(x, down, up, ids, scales, base)
    grads = torch.autograd.grad(out, leaves, case.grad.to(DEV))
    rng = _rng(11)
    for leaf, grad in zip(leaves, grads):
        flat, slope = leaf.detach().view(-1), grad.reshape(-1)
        for i in rng.choice(flat.numel(), 12, replace=False):
            kept = float(flat[i])
            sums = []
            for step in (1.0, -1.0):
                flat[i] = kept + step
                moved = bl.bitlogic_adapters(x.detach(), down.detach(), up.detach(), ids, scales,
                                             base)[0]
                sums.append((moved.double() * g).sum())
            flat[i] = kept
            # 24 x 18 outputs below 2^5 in size, each off by 40 roundings, times |grad| < 5
            assert abs(float(sums[0] - sums[1]) / 2 - float(slope[i])) < 432 * 32 * 5 * 40 * 2 ** -24


def test_no_rows_and_refusals():
    x, ids = torch.empty((0, 10), device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    down, up = torch.ones((3, 4, 10), device=DEV), torch.ones((3, 12, 4), device=DEV)
    out, hidden = bl.bitlogic_adapters(x, down, up, ids, want_hidden=True)
    assert out.shape == (0, 12) and hidden.shape == (0, 4)
    grads = bl.bitlogic_adapters_backward(out, x, hidden, down, up, ids)
    torch.cuda.synchronize()
    assert grads[0].shape == (0, 10) and not grads[1].any() and not grads[2].any()
    assert grads[1].shape == down.shape and grads[2].shape == up.shape
    leaf = down.clone().requires_grad_()
    bl.bitlogic_adapt(x, leaf, up, ids).sum().backward()
    assert not leaf.grad.any()
    x, ids = torch.ones((5, 10), device=DEV), torch.zeros(5, dtype=torch.int32, device=DEV)
    plan = bl.bitlogic_group_rows(ids, 3)
    for call, error, match in (
            (lambda: bl.bitlogic_adapters(x[:, :9], down, up, ids), ValueError, "columns"),
            (lambda: bl.bitlogic_adapters(x.half(), down, up, ids), TypeError, "beside"),
            (lambda: bl.bitlogic_adapters(x.int(), down.half(), up.half(), ids), TypeError,
             "beside"),
            (lambda: bl.bitlogic_adapters(x, down, up[:2].contiguous(), ids), ValueError, "up"),
            (lambda: bl.bitlogic_adapters(x, down, up, ids[:4]), ValueError, "ids has shape"),
            (lambda: bl.bitlogic_adapters(x, down, up, ids, torch.ones(2, device=DEV)),
             ValueError, "scales"),
            (lambda: bl.bitlogic_adapters(x, down, up, ids, base=x), ValueError, "base must"),
            (lambda: bl.bitlogic_adapters(x[:4], down, up, ids[:4], plan=plan), ValueError,
             "the plan is of 5 rows"),
            (lambda: bl.bitlogic_adapters(x, down[:2].contiguous(), up[:2].contiguous(), ids,
                                          plan=plan), ValueError, "the plan is of"),
            (lambda: bl.bitlogic_adapters_backward(x, x, None, down, up, ids), ValueError,
             "grad must"),
            (lambda: bl.bitlogic_adapters_backward(torch.ones((5, 12), device=DEV), x, None, down,
                                                   up, ids), bl.BitlogicError, "NULL"),
            (lambda: bl.bitlogic_adapters(x, down.expand(3, 4, 10).transpose(0, 1), up, ids),
             ValueError, "contiguous"),
            (lambda: bl.bitlogic_adapters(x[:, :10], torch.ones((3, 129, 10), device=DEV),
                                          torch.ones((3, 12, 129), device=DEV), ids),
             bl.BitlogicError, "rank 129")):
        with pytest.raises(error, match=match):
            call()


def test_streams_and_graphs():
    """Two captured passes with one plan and workspace, replayed in turn with eager work
    between; new ids make a new plan inside the graph."""
    cases = [Case((12,), 300, 150, 140, 10, 4, BF16) for _ in range(2)]
    other = Case((13,), 300, 600, 140, 10, 4, BF16)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    args = other.on()
    torch.cuda.synchronize()
    out, h = bl.bitlogic_adapters(*args, other.base_scale, want_hidden=True, stream=stream)
    grads = bl.bitlogic_adapters_backward(other.grad.to(DEV), args[0], h, *args[1:5],
                                          stream=stream)
    stream.synchronize()
    other.check(out, h)
    other.check_grads(*grads)
    room = torch.full((bl.load_library().bitlogic_group_rows_bytes(300, 4),), 255,
                      dtype=torch.uint8, device=DEV)
    workspace = torch.full((1 << 20,), 255, dtype=torch.uint8, device=DEV)
    held = []
    for case in cases:
        args, grad = case.on(), case.grad.to(DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            plan = bl.bitlogic_group_rows(args[3], 4, plan=room)
            out, h = bl.bitlogic_adapters(*args, case.base_scale, plan, want_hidden=True)
            grads = bl.bitlogic_adapters_backward(grad, args[0], h, *args[1:5], plan=plan,
                                                  workspace=workspace)
        held.append((graph, args, out, h, grads))
    rng = _rng(14)
    for turn in range(3):
        for case, (graph, args, out, h, grads) in zip(cases, held):
            case.ids = torch.from_numpy(rng.integers(-1, 4, 300).astype(np.int32))
            args[3].copy_(case.ids)
            graph.replay()
            torch.cuda.synchronize()
            case.check(out, h)
            case.check_grads(*grads)
            other.check(*other.run())


def test_backward_in_a_graph():
    """A captured training step with leaves of its own."""
    case = Case((15,), 200, 60, 50, 6, 3, F32)
    x, down, up, ids, scales, base = case.on()
    grad = case.grad.to(DEV)
    down.requires_grad_()
    up.requires_grad_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = bl.bitlogic_adapt(x, down, up, ids, scales, base, case.base_scale)
        grads = torch.autograd.grad(out, (down, up), grad)
    for turn in range(3):
        case.x = case.x * 0.5
        x.copy_(case.x)
        graph.replay()
        torch.cuda.synchronize()
        case.check(out)
        case.check_grads(None, *grads)


# ------------------------------------------------------------ rows by group

def _check_plan(ids, n_groups):
    """The order and starts in a plan, which its layout puts first."""
    groups = bl.bitlogic_group_rows(ids.to(DEV), n_groups)
    torch.cuda.synchronize()
    n = len(ids)
    order, starts = oracle.groups(ids.numpy(), n_groups)
    words = groups.plan.cpu()[:groups.plan.numel() // 4 * 4].view(torch.int32).numpy()
    assert np.array_equal(words[:n], order)
    at = (n + 63) // 64 * 64
    assert np.array_equal(words[at:at + n_groups + 2], starts)


@pytest.mark.parametrize("n,g", [(1, 1), (63, 3), (64, 2), (65, 70), (1000, 1), (1024, 16),
                                 (5000, 1100), (8192, 4096), (8193, 5), (30000, 200),
                                 (100000, 4096), (300001, 33)])
def test_rows_by_group(n, g):
    rng = _rng(16, n, g)
    _check_plan(torch.from_numpy(rng.integers(-2, g + 2, n).astype(np.int32)), g)
    few = rng.choice(g, min(g, 3))
    _check_plan(torch.from_numpy(few[rng.integers(0, len(few), n)].astype(np.int32)), g)
    _check_plan(torch.full((n,), -1, dtype=torch.int32), g)
    _check_plan(torch.full((n,), g - 1, dtype=torch.int32), g)


def test_more_rows_than_a_run_a_wave():
    """Past 2^20 rows a wave's run is longer than 1024 rows; rows of two columns."""
    n = (1 << 20) + 4097
    rng = _rng(18)
    ids = torch.from_numpy(rng.integers(0, 9, n).astype(np.int32))
    _check_plan(ids, 9)
    case = Case((18,), 50, 2, 3, 1, 9, F32)
    x = _normal(rng, (n, 2), F32).to(DEV)
    _, down, up, _, scales, _ = case.on()
    out, h = bl.bitlogic_adapters(x, down, up, ids.to(DEV), scales, want_hidden=True)
    at = ids.long().to(DEV)
    want_h = (down.double()[at] * x.double()[:, None]).sum(2)
    want = scales.double()[at][:, None] * (up.double()[at] * want_h[:, None]).sum(2)
    assert ((out.double() - want).abs() <= 2.0 ** -20 * (want.abs() + 10)).all()
    grads = bl.bitlogic_adapters_backward(torch.ones_like(out), x, h, down, up, ids.to(DEV),
                                          scales)
    back = up.double().sum(1)                             # [9][1]
    for a in range(9):
        rows = x.double()[at == a]
        # n / 9 terms of size up to 10: roundings of a running sum
        want_d = scales[a].double() * back[a] * rows.sum(0)
        size = float((scales[a].double() * back[a].abs() * rows.abs().sum(0)).max())
        assert ((grads[1][a].double() - want_d).abs() <= size * 2.0 ** -24 * 8192).all()


def _far(n, c, dtype, step):
    """Rows [n][c], `step` elements apart, in memory that holds anything between them."""
    return torch.empty((n - 1) * step + c, dtype=dtype, device=DEV).as_strided((n, c), (step, 1))


@pytest.mark.parametrize("f,c,rank", [(100, 120, 8), (301, 403, 24)])
def test_rows_past_32_bit_offsets(f, c, rank):
    """Rows 2^26 elements apart, narrow and wide, both passes: the same as of rows together."""
    rng = np.random.default_rng(f)
    n, g, dtype, step = 70, 3, torch.bfloat16, 1 << 26    # 9.4 GB a tensor
    of = lambda *s: torch.from_numpy(rng.normal(0, 0.3, s).astype(np.float32)).to(DEV, dtype)  # noqa: E731,E501
    x, base, grad, down, up = of(n, f), of(n, c), of(n, c), of(g, rank, f), of(g, c, rank)
    ids = torch.from_numpy(rng.integers(-1, g, n).astype(np.int32)).to(DEV)
    plan = bl.bitlogic_group_rows(ids, g)
    want, hidden = bl.bitlogic_adapters(x, down, up, ids, 0.5, base, 1.0, plan, want_hidden=True)
    want_grads = bl.bitlogic_adapters_backward(grad, x, hidden, down, up, ids, 0.5, plan)
    far_x, far_out, far_grad = (_far(n, t.shape[1], dtype, step) for t in (x, base, grad))
    for far, near in ((far_x, x), (far_out, base), (far_grad, grad)):
        far.copy_(near)
    got, far_hidden = bl.bitlogic_adapters(far_x, down, up, ids, 0.5, far_out, 1.0, plan,
                                           out=far_out, want_hidden=True)
    assert torch.equal(got, want) and torch.equal(far_hidden, hidden)
    grads = bl.bitlogic_adapters_backward(far_grad, far_x, far_hidden, down, up, ids, 0.5, plan,
                                          grad_x=_far(n, f, dtype, step))
    for a, b in zip(grads, want_grads):
        assert torch.equal(a, b)


def test_adapters_past_32_bit_offsets():
    """The last of nine adapters of 512 MB each."""
    rng = np.random.default_rng(8)
    g, rank, f, c = 9, 128, 1 << 20, 10
    down = torch.zeros(g, rank, f, device=DEV)
    at = torch.from_numpy(np.sort(rng.choice(f, 5, replace=False))).to(DEV)
    down[8, :, at] = torch.from_numpy(rng.normal(size=(rank, 5)).astype(np.float32)).to(DEV)
    up = torch.from_numpy(rng.normal(size=(g, c, rank)).astype(np.float32)).to(DEV)
    x = torch.zeros(40, f, device=DEV)
    x[:, at] = torch.from_numpy(rng.normal(size=(40, 5)).astype(np.float32)).to(DEV)
    ids = torch.full((40,), 8, dtype=torch.int32, device=DEV)
    d5, x5, u = (t.double().cpu() for t in (down[8][:, at], x[:, at], up[8]))
    want = x5 @ d5.t() @ u.t()
    size = x5.abs() @ d5.abs().t() @ u.abs().t()
    for plan in (bl.bitlogic_group_rows(ids, g), None):
        rows = slice(None) if plan else slice(0, 20)
        got, _ = bl.bitlogic_adapters(x[rows], down, up, ids[rows], 1.0, plan=plan)
        # five terms that are not zero, then 128: a rounding each, in 32 bits
        assert ((got.double().cpu() - want[rows]).abs() <= 140 * 2.0 ** -24 * size[rows]).all()


def test_plan_written_again_before_the_backward_pass_is_refused():
    case = Case((20,), 100, 60, 50, 6, 3, F32)
    x, down, up, ids, scales, base = case.on()
    for leaf in (x, down, up):
        leaf.requires_grad_()
        plan = bl.bitlogic_group_rows(ids, 3)
        out = bl.bitlogic_adapt(x, down, up, ids, scales, base, case.base_scale, plan)
        again = bl.bitlogic_group_rows((ids + 1) % 3, 3, plan=plan.plan)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            torch.autograd.grad(out, leaf, case.grad.to(DEV))
        # the plan written again serves calls from then on
        case.ids, first = (case.ids + 1) % 3, case.ids
        out = bl.bitlogic_adapt(x, down, up, (ids + 1) % 3, scales, base, case.base_scale, again)
        case.check(out)
        grad, = torch.autograd.grad(out, leaf, case.grad.to(DEV))
        case.check_grads(*(grad if v is leaf else None for v in (x, down, up)))
        case.ids = first
        leaf.requires_grad_(False)


def test_outputs_over_inputs_are_refused():
    """The gradient of x over the gradient of out, which the weights' gradients still read; or
    between its rows, where nothing is lost."""
    for f in (60, 700):
        case = Case((21,), 50, f, f, 6, 3, F32)
        x, down, up, ids, scales, base = case.on()
        _, hidden = bl.bitlogic_adapters(x, down, up, ids, scales, base, case.base_scale,
                                         want_hidden=True)
        wide = torch.zeros((50, 2 * f), device=DEV)
        grad, grad_x = wide[:, :f], wide[:, f:]
        grad.copy_(case.grad)
        case.check_grads(*bl.bitlogic_adapters_backward(grad, x, hidden, down, up, ids, scales,
                                                        grad_x=grad_x))
        for over in (grad, wide[:, 1:f + 1], x):
            with pytest.raises(bl.BitlogicError, match="overlaps"):
                bl.bitlogic_adapters_backward(grad, x, hidden, down, up, ids, scales, grad_x=over)
        with pytest.raises(bl.BitlogicError, match="grad_down overlaps down"):
            bl.bitlogic_adapters_backward(grad, x, hidden, down, up, ids, scales, grad_down=down)
        with pytest.raises(bl.BitlogicError, match="hidden overlaps base"):
            bl.bitlogic_adapters(x, down, up, ids, scales, base,
                                 hidden=base.view(-1)[:300].view(50, 6))
        assert torch.equal(grad, case.grad.to(DEV))


@pytest.mark.parametrize("type_", [F32, BF16])
@pytest.mark.parametrize("n", [20, 33, 300])
def test_rows_are_grouped_once_for_both_passes(n, type_, monkeypatch):
    """Whichever gradients are asked for; and the backward pass has the forward pass's rows."""
    case = Case((22,), n, 60, 50, 6, 3, type_)
    x, down, up, ids, scales, base = case.on()
    calls, group = [], bl.bitlogic_group_rows
    monkeypatch.setattr(bl, "bitlogic_group_rows",
                        lambda *a, **k: calls.append(1) or group(*a, **k))
    leaves = (x, down, up)
    for wanted in ((x,), (down,), (up,), leaves):
        for leaf in wanted:
            leaf.requires_grad_()
        calls.clear()
        alone = n <= 32 and len(wanted) == 1 and wanted[0] is x
        own = ids.clone()
        out = bl.bitlogic_adapt(x, down, up, own, scales, base, case.base_scale)
        if n > 32:
            own.data.fill_(1)                             # (no version of it moves)
        grads = dict(zip(map(id, wanted), torch.autograd.grad(out, wanted, case.grad.to(DEV))))
        assert len(calls) == (not alone)
        case.check(out)
        case.check_grads(*(grads.get(id(v)) for v in leaves))
        for leaf in wanted:
            leaf.requires_grad_(False)
    calls.clear()
    base.requires_grad_()
    out = bl.bitlogic_adapt(x, down, up, ids, scales, base, case.base_scale)
    torch.autograd.grad(out, base, case.grad.to(DEV))
    assert len(calls) == (n > 32)


@pytest.mark.parametrize("f,c,r,rows", [(2, 3, 1, 1024), (70, 60, 3, 4096)])
def test_gradients_of_more_rows_than_a_run_a_wave(f, c, r, rows):
    """All three past 2^20 rows, in chunks of either cut.  Every value is positive, so that a
    chunk that is lost or counted twice is a hundredth of the sum."""
    n, g = (1 << 20) + 4097, 9
    gen = torch.Generator(DEV).manual_seed(19)
    of = lambda *s: 0.5 + torch.rand(s, device=DEV, generator=gen)              # noqa: E731
    x, grad, down, up, scales = of(n, f), of(n, c), of(g, r, f), of(g, c, r), of(g)
    ids = torch.randint(-1, g, (n,), device=DEV, generator=gen).int()
    _, hidden = bl.bitlogic_adapters(x, down, up, ids, scales, want_hidden=True)
    got = bl.bitlogic_adapters_backward(grad, x, hidden, down, up, ids, scales)
    x, grad, down, up, scales = (v.double() for v in (x, grad, down, up, scales))
    # roundings of the terms, of a chunk's sum, and of the sum over a group's chunks
    own = (f + c + r + 8) * 2.0 ** -24
    off = own + (rows + n // rows) * 2.0 ** -24
    assert off < 0.1 * rows / (n / g)                     # a tenth of a chunk
    assert not got[0][ids < 0].any()
    for a in range(g):
        at = (ids == a).nonzero()[:, 0]
        xa, ga = x[at], grad[at]
        back, h = ga @ up[a], xa @ down[a].t()
        for value, want, bound in (
                (got[0][at], scales[a] * (back @ down[a]), own),
                (got[1][a], scales[a] * (back.t() @ xa), off),
                (got[2][a], scales[a] * (ga.t() @ h), off)):
            assert ((value.double() - want).abs() <= bound * want).all()


def test_given_outputs_count_as_changed():
    """What autograd has kept of a tensor that a call then writes is refused, not wrong."""
    case = Case((23,), 40, 60, 60, 6, 3, F32)
    x, down, up, ids, scales, base = case.on()
    leaf = torch.ones((40, 60), device=DEV, requires_grad=True)
    narrow = torch.ones((40, 6), device=DEV, requires_grad=True)
    hidden = torch.ones((40, 6), device=DEV)

    def backward(name, shape):
        kept = torch.ones(shape, device=DEV, requires_grad=True)
        y = kept.exp()
        bl.bitlogic_adapters_backward(case.grad.to(DEV), x, hidden, down, up, ids, scales,
                                      **{name: y.detach()})
        return kept, y

    y = leaf.exp()                                        # keeps its result
    bl.bitlogic_adapters(x, down, up, ids, scales, y.detach(), out=y.detach())
    h = narrow.exp()
    bl.bitlogic_adapters(x, down, up, ids, scales, hidden=h.detach())
    d = leaf.exp()
    bl.bitlogic_dropout(d.detach(), 0.5, 1, out=d.detach())
    made = [(leaf, y), (narrow, h), (leaf, d)]
    made += [backward(name, shape) for name, shape in
             (("grad_x", x.shape), ("grad_down", down.shape), ("grad_up", up.shape))]
    for kept, value in made:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            torch.autograd.grad(value.sum(), kept)
