"""Draft verification against the 64-bit oracle: every pair of element types, class counts on
both sides of each form's limits, lengths from none to many, masks, ties, greedy requests,
numbers next to a decision's border, strides, streams and graphs.

Accepted drafts and tokens are those of 64-bit arithmetic and compared exactly (inputs whose
decision 64 bits leave open do not occur: equal masses have equal roundings).  A
log-probability comes from a sum of 32-bit terms: terms are off by at most 2.5 |x| 2^-24 and
what is far below the largest has no weight, so within REL = 1e-5, and 2^-22 of itself."""
import numpy as np
import pytest
import torch

import draft_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
REL = 1e-5
FLOATS = [torch.float32, torch.float16, torch.bfloat16]
TYPES = [torch.int32] + FLOATS
SIZES = [1, 2, 10, 16, 37, 100, 257, 1000, 1025, 4095, 4096, 4097, 8192, 8199, 32003, 131075]


def _rng(*key):
    return np.random.default_rng([7, *[int(k) for k in key]])


def _logits(rng, shape, dtype, spread=2.0):
    x = rng.normal(0, spread, shape)
    if dtype == torch.int32:
        return torch.from_numpy(np.round(20 * x + 320).astype(np.int32))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def _host(t):
    x = t.detach().cpu()
    x = x.double().numpy() if x.dtype != torch.int32 else x.numpy().astype(np.float64)
    return x, np.isnan(x) | (x == (-2.0 ** 31 if t.dtype == torch.int32 else -np.inf))


def _gumbel(rng, *shape):
    return torch.from_numpy(rng.gumbel(size=shape).astype(np.float32))


class Case:
    """Inputs of a call, on the host; t, tq: numbers or float32 tensors."""

    def __init__(self, rng, r, d, c, type_=torch.float32, draft_type=torch.float32, t=None,
                 tq=None, lengths=None, near=0.7):
        self.x = _logits(rng, (r, d + 1, c), type_)
        scale = 20.0 if type_ == torch.int32 else 1.0
        self.t = scale if t is None else t
        self.y = None
        y = self.x[:, :d].double() / scale + torch.from_numpy(near * rng.normal(size=(r, d, c)))
        scale_q = 20.0 if draft_type == torch.int32 else 1.0
        self.tq = scale_q if tq is None else tq
        if draft_type is not None:
            self.y = (y * scale_q).round().int() if draft_type == torch.int32 \
                else y.to(draft_type)
        seen = (y if self.y is None else self.y.double() / scale_q).numpy()
        self.drafted = torch.from_numpy(
            (seen + rng.gumbel(size=seen.shape)).argmax(2).astype(np.int32)) if d \
            else torch.zeros((r, 0), dtype=torch.int32)
        self.uniform = torch.from_numpy(rng.random((r, d)).astype(np.float32))
        self.noise = _gumbel(rng, r, c)
        self.lengths = lengths

    def run(self, **kw):
        on = lambda v: v.to(DEV) if torch.is_tensor(v) else v                    # noqa: E731
        got = bl.bitlogic_verify(on(self.x), on(self.drafted), on(self.y), on(self.uniform),
                                 on(self.noise), on(self.lengths), on(self.t), on(self.tq), **kw)
        torch.cuda.synchronize()
        return got

    def want(self):
        r, d = self.drafted.shape
        x, masked = _host(self.x)
        y, y_masked = (None, None) if self.y is None else _host(self.y)
        of = lambda v, i: float(v[i]) if torch.is_tensor(v) else float(v)        # noqa: E731
        out = []
        for i in range(r):
            n = d if self.lengths is None else min(max(int(self.lengths[i]), 0), d)
            out.append(oracle.verify(
                x[i], masked[i], self.drafted[i, :n].numpy(), None if y is None else y[i],
                None if y is None else y_masked[i], self.uniform[i].numpy().astype(np.float64),
                self.noise[i].numpy().astype(np.float64), of(self.t, i), of(self.tq, i)))
        return out

    def check(self, got=None):
        accepted, token, log_prob = (v.cpu().numpy() for v in (got or self.run()))
        want = self.want()
        assert accepted.tolist() == [w[0] for w in want]
        assert token.tolist() == [w[1] for w in want]
        exact = np.array([w[2] for w in want])
        fine = np.isfinite(exact)
        assert np.array_equal(log_prob[~fine], exact[~fine].astype(np.float32))
        off = np.abs(log_prob[fine] - exact[fine])
        assert (off <= REL + 2.0 ** -22 * np.abs(exact[fine])).all()
        return want


def _requests(c):
    return 21 if c <= 1025 else 5


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", SIZES)
def test_sizes(c, dtype):
    rng = _rng(1, c, TYPES.index(dtype))
    r = _requests(c)
    lengths = torch.from_numpy(rng.integers(-1, 6, r).astype(np.int32))
    Case(rng, r, 4, c, dtype, dtype).check()
    Case(rng, r, 4, c, dtype, dtype, lengths=lengths).check()
    Case(rng, r, 3, c, dtype, None).check()


@pytest.mark.parametrize("draft_type", TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [100, 5003])
def test_pairs_of_types(c, dtype, draft_type):
    rng = _rng(2, c, TYPES.index(dtype), TYPES.index(draft_type))
    Case(rng, 9, 3, c, dtype, draft_type).check()


@pytest.mark.parametrize("r,d,c", [(1, 0, 50), (3, 0, 9000), (1, 1, 20000), (2, 70, 40),
                                   (2, 70, 4500), (1, 130, 4500), (150, 5, 4097), (400, 1, 5003),
                                   (1300, 2, 33), (700, 0, 4500), (260, 3, 6001)])
def test_requests_and_lengths(r, d, c):
    rng = _rng(3, r, d, c)
    case = Case(rng, r, d, c, torch.bfloat16, torch.bfloat16, near=0.2,
                lengths=torch.from_numpy(rng.integers(0, d + 1, r).astype(np.int32)))
    want = case.check()
    if d >= 70:                       # long walks among them
        case.uniform[:] = 0.0
        case.lengths[:] = d
        want = case.check()
        assert max(w[0] for w in want) > 64


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [40, 1500, 7001])
def test_masks_and_greedy(c, dtype):
    rng = _rng(4, c, TYPES.index(dtype))
    r, d = 26, 3
    case = Case(rng, r, d, c, dtype, dtype)
    scale = case.t
    low = torch.iinfo(dtype).min if dtype == torch.int32 else -np.inf
    x, y = case.x, case.y
    x[0] = low                                            # nothing in the rows
    x[1, 0] = low
    x[2, 1] = low
    x[2, 1, c // 2] = 3                                   # one class
    case.drafted[2, 0] = int(x[2, 0].double().argmax())
    y[3] = low                                            # a drafter that rules all out
    y[4, 0, case.drafted[4, 0]] = low                     # and one that rules its draft out
    x[5, 0, case.drafted[5, 0]] = low
    x[6] = 7                                              # all equal
    y[6] = 9
    case.drafted[7, 0], case.drafted[8, 1] = -1, c        # no classes
    x[9, :, ::2] = low
    y[9, :, 1::2] = low                                   # nothing in common
    case.uniform[10] = 1.0                                # just past the range
    case.noise[11] = -np.inf
    case.noise[12] = np.nan
    case.noise[13, ::3] = np.inf                          # the lowest of equals
    x[14, :d] = y[14]                                     # p = q: all stand
    x[15] = torch.round(x[15].double() / 16).to(dtype)    # few values
    if dtype != torch.int32:
        x[16, 0, ::3] = np.nan
        y[16, 0, 1::3] = np.nan
        x[17] = torch.finfo(dtype).min                    # masks of the lowest value
        x[17, :, c // 3] = -torch.finfo(dtype).max / 2
        x[18, :, c // 4] = np.inf
        y[18, 0, c // 4] = np.inf
        y[19, 0, c // 5] = np.inf
        x[20] = torch.where(torch.arange(c) % 2 == 0, 0.0, -0.0)
    else:
        x[16, 0, c // 3], x[16, 0, c // 3 + 1] = 2 ** 31 - 1, 2 ** 31 - 2
        x[17] = 2 ** 30 + torch.arange(c, dtype=torch.int32) % 3        # above 2^24
    t = torch.full((r,), scale)
    tq = torch.full((r,), scale)
    t[21], t[22], tq[23], tq[24] = 0.0, -1.0, 0.0, -2.0
    t[25], tq[25] = 0.03 * scale, 0.02 * scale
    case.check()
    case.t, case.tq = t, tq
    case.check()
    case.t = torch.zeros(r)
    case.check()
    case.t = 0.0
    case.noise, noise = None, case.noise                  # greedy alone needs no numbers
    got = case.run()
    case.noise = noise
    case.check(got)


def test_extreme_temperatures():
    rng = _rng(5)
    for c in (60, 5000):
        case = Case(rng, 8, 2, c)
        case.t = torch.tensor([1e-40, 1e-30, 1e-10, 1e10, 3e38, np.inf, 0.5, 1e-3])
        case.tq = case.t.flip(0).clone()
        accepted, token, log_prob = case.run()
        case.t = case.t.clamp(2.0 ** -126, torch.finfo(torch.float32).max)
        case.tq = case.tq.clamp(2.0 ** -126, torch.finfo(torch.float32).max)
        case.check((accepted, token, log_prob))


@pytest.mark.parametrize("c,r", [(37, 40), (700, 24), (4500, 10), (4500, 200)])
def test_numbers_next_to_a_border(c, r):
    """uniform numbers on either side of p / q by a rounding: sums in 32 bits could not tell."""
    rng = _rng(6, c, r)
    d = 2
    case = Case(rng, r, d, c, torch.float32, torch.float32, near=0.5)
    x, masked = _host(case.x)
    y, y_masked = _host(case.y)
    for i in range(r):
        for k in range(d):
            log_p, _ = oracle.shares(x[i, k], masked[i, k], 1.0)
            log_q, _ = oracle.shares(y[i, k], y_masked[i, k], 1.0)
            t = int(case.drafted[i, k])
            ratio = np.exp(log_p[t] - log_q[t])
            u = np.float32(ratio)
            side = 1 if (i + k) % 3 else -1               # most stand, by a rounding
            while (float(u) < ratio) != (side == 1):
                u = np.nextafter(u, np.float32(-side * 9))
            case.uniform[i, k] = float(u)
    want = case.check()
    assert {w[0] for w in want} == {0, 1, 2}


@pytest.mark.parametrize("c", [37, 700, 4500, 30011])
def test_draws_next_to_a_border(c):
    """Two classes whose masses times their numbers are equal but for a rounding, their
    masses small differences of nearly equal p and q."""
    rng = _rng(7, c)
    r = 16
    case = Case(rng, r, 1, c, torch.float32, torch.float32, near=0.01)
    case.uniform[:] = 0.9999999                           # 1 - 2^-23.2: rejected where p < q
    x, _ = _host(case.x)
    y, _ = _host(case.y)
    none = np.zeros(c, bool)
    for i in range(r):
        log_p, _ = oracle.shares(x[i, 0], none, 1.0)
        log_q, _ = oracle.shares(y[i, 0], none, 1.0)
        mass = np.exp(log_p) - np.exp(log_q)
        case.drafted[i, 0] = int(mass.argmin())
        a, b = rng.choice(np.nonzero(mass > 0)[0], 2, replace=False)
        noise = case.noise[i].numpy()
        noise[a] = 60.0 - np.log(mass[a])
        noise[b] = np.float32(np.log(mass[a]) + float(noise[a]) - np.log(mass[b]))
        if i % 2:
            noise[b] = np.nextafter(noise[b], np.float32(-99 if i % 4 == 1 else 999))
    want = case.check()
    assert all(w[0] == 0 for w in want)


def test_strides_outputs_and_alignment():
    rng = _rng(8)
    for c in (50, 4500):
        for dtype in TYPES:
            r, d = 6, 3
            case = Case(rng, r, d, c, dtype, dtype)
            want = case.run()
            wide = torch.zeros((r, d + 2, c + 7), dtype=dtype)
            wide[:, 1:, 3:c + 3] = case.x
            wide_q = torch.zeros((d, r, c + 1), dtype=dtype)
            wide_q[:, :, 1:] = case.y.transpose(0, 1)
            noise = torch.zeros((r, c + 5))
            noise[:, 5:] = case.noise
            outs = dict(accepted=torch.empty(r, dtype=torch.int32, device=DEV),
                        token=torch.empty(r, dtype=torch.int32, device=DEV))
            got = bl.bitlogic_verify(
                wide.to(DEV)[:, 1:, 3:c + 3], case.drafted.to(DEV),
                wide_q.to(DEV)[:, :, 1:].transpose(0, 1), case.uniform.to(DEV),
                noise.to(DEV)[:, 5:], temperature=case.t, draft_temperature=case.tq,
                want_log_prob=False, **outs)
            assert got[0] is outs["accepted"] and got[1] is outs["token"] and got[2] is None
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            # one row of logits for all requests and drafts
            case.x = case.x[:1, :1].expand(r, d + 1, c)
            case.y = case.y[:1, :1].expand(r, d, c)
            got = bl.bitlogic_verify(
                case.x[:1, :1].to(DEV).expand(r, d + 1, c), case.drafted.to(DEV),
                case.y[:1, :1].to(DEV).expand(r, d, c), case.uniform.to(DEV),
                case.noise.to(DEV), temperature=case.t, draft_temperature=case.tq)
            case.check(got)


def test_no_requests_and_refusals():
    empty = torch.empty((0, 4, 10), device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    got = bl.bitlogic_verify(empty, torch.empty((0, 3), **i32), empty[:, :3],
                             torch.empty((0, 3), device=DEV), torch.empty((0, 10), device=DEV))
    assert all(v.shape == (0,) for v in got)
    x = torch.zeros((2, 4, 10), device=DEV)
    u, z, t = torch.zeros((2, 3), device=DEV), torch.zeros((2, 10), device=DEV), \
        torch.zeros((2, 3), **i32)
    with pytest.raises(ValueError, match="drafted must be contiguous"):
        bl.bitlogic_verify(x, t[:, :2], x[:, :3], u, z)
    with pytest.raises(ValueError, match="drafted has shape"):
        bl.bitlogic_verify(x, t[:, :2].contiguous(), x[:, :3], u, z)
    with pytest.raises(ValueError, match="draft_logits has shape"):
        bl.bitlogic_verify(x, t, x, u, z)
    with pytest.raises(ValueError, match="noise must be"):
        bl.bitlogic_verify(x, t, x[:, :3], u, z[:, :9])
    with pytest.raises(TypeError, match="drafted has dtype"):
        bl.bitlogic_verify(x, t.long(), x[:, :3], u, z)
    with pytest.raises(bl.BitlogicError, match="NULL"):
        bl.bitlogic_verify(x, t, x[:, :3], u, None)
    with pytest.raises(ValueError, match="a row more"):
        bl.bitlogic_verify(x[:, :0], t, x[:, :0], u, z)


@pytest.mark.parametrize("r,c", [(30, 100), (3, 20000), (130, 5003)])
def test_streams_and_graphs(r, c):
    """Two captured calls that share a workspace, replayed in turn with eager work between;
    a call on another stream."""
    rng = _rng(9, r, c)
    cases = [Case(rng, r, 4, c, torch.bfloat16, torch.bfloat16) for _ in range(2)]
    other = Case(rng, r, 4, c, torch.bfloat16, torch.bfloat16)
    need = bl.load_library().bitlogic_verify_workspace_bytes(r, 4, c)
    workspace = torch.full((max(need, 8),), 255, dtype=torch.uint8, device=DEV)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        other.check(other.run(workspace=workspace))
    got = other.run(stream=stream)
    other.check(got)
    held = []
    for case in cases:
        args = [v.to(DEV) for v in (case.x, case.drafted, case.y, case.uniform, case.noise)]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = bl.bitlogic_verify(*args, temperature=case.t, draft_temperature=case.tq,
                                     workspace=workspace)
        held.append((graph, args, out))
    for turn in range(3):
        for case, (graph, args, out) in zip(cases, held):
            case.noise = _gumbel(rng, r, c)
            args[4].copy_(case.noise)
            graph.replay()
            torch.cuda.synchronize()
            case.check(out)
            other.run(workspace=workspace)


@pytest.mark.parametrize("r,d,c", [(300, 2, 5003), (350, 2, 64001)])
def test_shares_far_below_the_largest(r, d, c):
    """Drafts whose shares are e^-100000 in both rows: their exponents cancel, and what 32 bits
    would leave of the difference must not reject a draft and have the rows behind it left out."""
    rng = np.random.default_rng(12)
    t = 0.01
    x, y = np.zeros((r, d + 1, c), np.float32), np.zeros((r, d, c), np.float32)
    drafted = rng.integers(1, c, (r, d)).astype(np.int32)
    at = np.arange(r)[:, None], np.arange(d)[None], drafted
    x[at] = -rng.uniform(900, 1100, (r, d))
    y[at] = x[at] + rng.uniform(0, 0.02, (r, d)).astype(np.float32)
    # the sums are the same classes in both rows: p / q = e^((x - y) / T)
    ratio = np.exp((x[at].astype(np.float64) - y[at]) / float(np.float32(t)))
    uniform = (ratio * 0.9995).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).to(DEV)           # noqa: E731
    accepted, token, _ = bl.bitlogic_verify(dev(x), dev(drafted), dev(y), dev(uniform),
                                            _gumbel(rng, r, c).to(DEV), temperature=t)
    assert (accepted == d).all() and ((token >= 0) & (token < c)).all()


@pytest.mark.parametrize("near", [0.3, 2.0])
@pytest.mark.parametrize("r,d,c", [(330, 3, 1500), (460, 2, 4000), (460, 2, 4096), (256, 3, 8193),
                                   (350, 2, 64001)])
def test_many_requests(r, d, c, near):
    """Requests enough for a wave each, or a block a row; drafts that stand and that do not."""
    rng = _rng(13, r, c, 10 * near)
    lengths = torch.from_numpy(rng.integers(0, d + 1, r).astype(np.int32))
    case = Case(rng, r, d, c, torch.bfloat16, torch.bfloat16, lengths=lengths, near=near)
    # rows of masks, masked drafts, requests without randomness
    case.x[5, 0] = float("-inf")
    case.y[6, 0] = float("-inf")
    case.x[torch.arange(7, 30), 0, case.drafted[7:30, 0].long()] = float("-inf")
    case.t = torch.from_numpy(np.where(np.arange(r) % 9 == 4, 0, 0.8).astype(np.float32))
    want = case.check()
    assert len({w[0] for w in want}) > 1


@pytest.mark.parametrize("c,r", [(1500, 330), (4000, 460)])
def test_many_numbers_next_to_a_border(c, r):
    test_numbers_next_to_a_border(c, r)


@pytest.mark.parametrize("c", [100, 5003])
def test_requests_past_32_bit_offsets(c):
    """Requests 2^30 elements apart, on both sides, and numbers 2^28: as of requests together."""
    rng = _rng(14, c)
    r, d = 5, 2
    case = Case(rng, r, d, c, torch.bfloat16, torch.bfloat16)

    def far(t, step):                                     # up to 8.6 GB a tensor
        size = (r - 1) * step + t[0].numel()
        strides = (step, c, 1) if t.dim() == 3 else (step, 1)
        out = torch.empty(size, dtype=t.dtype, device=DEV).as_strided(t.shape, strides)
        return out.copy_(t)

    got = bl.bitlogic_verify(far(case.x, 1 << 30), case.drafted.to(DEV), far(case.y, 1 << 30),
                             case.uniform.to(DEV), far(case.noise, 1 << 28),
                             temperature=case.t, draft_temperature=case.tq)
    case.check(got)


@pytest.mark.parametrize("dtype", [torch.int32, torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,d,c", [(350, 2, 64001), (600, 1, 60001)])
def test_drafters_rows_without_mass_among_many_long_ones(r, d, c, dtype):
    """A draft that the drafter itself rules out with its whole row has p / q = infinity and
    stands: the rows behind it count, whatever the workspace held before."""
    rng = _rng(15, r, c, TYPES.index(dtype))
    case = Case(rng, r, d, c, dtype, dtype)
    low = torch.iinfo(dtype).min if dtype == torch.int32 else -np.inf
    case.y[:, 0] = low
    if dtype != torch.int32:
        case.y[::2, 0] = np.nan
    want = case.want()
    case.want = lambda: want
    need = bl.load_library().bitlogic_verify_workspace_bytes(r, d, c)
    for fill in (0, 63):                                  # (63: small positive numbers)
        workspace = torch.full((need,), fill, dtype=torch.uint8, device=DEV)
        case.check(case.run(workspace=workspace))
    assert {w[0] for w in want} >= set(range(1, d + 1))


@pytest.mark.parametrize("r,d,c", [(256, 3, 65537), (400, 2, 60003)])
def test_shares_far_below_the_largest_a_block_a_row(r, d, c):
    test_shares_far_below_the_largest(r, d, c)


@pytest.mark.parametrize("near", [0.3, 2.0])
def test_many_requests_a_block_a_row(near):
    test_many_requests(256, 3, 65537, near)


def _ramp(c, t, dtype):
    """A row of c classes that ascends from 0 to 1 (int32: from 0 to c - 1), every value exact, a
    temperature for it, and log p: each lane's maximum grows with every load."""
    x = torch.arange(c, dtype=torch.int32)
    if dtype == torch.float32:
        x, scale = x.float() / c, 1.0
    else:
        scale = float(c)
    t = float(np.float32(t * scale))
    y = x.double().numpy() / t
    return x, t, y - y[-1] - np.log(np.exp(y - y[-1]).sum())


RAMP_T = [0.7, 0.9, 1.0, 1.3, 1.4]


@pytest.mark.parametrize("dtype", [torch.float32, torch.int32])
@pytest.mark.parametrize("c,r", [(2048, 400), (3900, 480), (1 << 17, 30), (1 << 20, 500),
                                 (1 << 22, 500), (1 << 22, 600), (1 << 22, 10)])
def test_ascending_rows(c, r, dtype):
    """Rows along which a lane's sum is made relative to a larger logit again and again, against
    a flat drafter: numbers from 4e-5 below p / q to 4e-5 above it."""
    rng = _rng(16, c, r, TYPES.index(dtype))
    t_of = torch.empty(r)
    draft, noise = c // 4, _gumbel(rng, 1, c)
    z = noise[0].double().numpy()
    uniform, want = torch.empty(r, 1), []
    for k, t in enumerate(RAMP_T):
        x, t_of[k::5], log_p = _ramp(c, t, dtype)
        t = float(t_of[k])
        ratio = np.exp(log_p[draft] + np.log(c))
        stands = int((log_p + z).argmax())
        with np.errstate(divide="ignore"):
            drawn = int((np.log(np.maximum(np.exp(log_p) - 1 / c, 0)) + z).argmax())
        rows = range(k, r, 5)
        for n, i in enumerate(rows):
            uniform[i] = ratio * (1 + (2 * (n + 0.5) / len(rows) - 1) * 4e-5)
            ok = float(uniform[i]) < ratio
            want.append((i, int(ok), stands if ok else drawn, log_p[stands if ok else drawn]))
    x = x.to(DEV).expand(r, 2, c)
    flat = torch.zeros(c, device=DEV).expand(r, 1, c)
    accepted, token, log_prob = (v.cpu().numpy() for v in bl.bitlogic_verify(
        x, torch.full((r, 1), draft, dtype=torch.int32, device=DEV), flat, uniform.to(DEV),
        noise.to(DEV).expand(r, c), temperature=t_of.to(DEV)))
    at = [w[0] for w in want]
    assert accepted[at].tolist() == [w[1] for w in want]
    assert token[at].tolist() == [w[2] for w in want]
    off = np.abs(log_prob[at] - np.array([w[3] for w in want]))
    assert (off <= REL + 2.0 ** -22 * 40).all()


@pytest.mark.parametrize("c,r", [(1 << 17, 100), (1 << 20, 505), (1 << 22, 505)])
def test_draws_from_ascending_rows(c, r):
    """Two classes whose scores are within 2.5e-3 of each other, one of them with a mass that is a
    fiftieth of its p: what its row's sum is off by counts fifty times."""
    noise = torch.full((r, c), -1000.0, device=DEV)
    t_of, want = torch.empty(r), []
    for k, t in enumerate(RAMP_T):
        x, t_of[k::5], log_p = _ramp(c, t, torch.float32)
        t = float(t_of[k])
        delta = -np.log(c) - log_p                        # log q - log p, falling
        a, b = int(np.searchsorted(-delta, 0.02)), c - 1
        score = lambda i: log_p[i] + np.log(-np.expm1(delta[i]))                 # noqa: E731
        rows = range(k, r, 5)
        for n, i in enumerate(rows):
            z = np.float32(score(b) - score(a) + (2 * (n + 0.5) / len(rows) - 1) * 2.5e-3)
            noise[i, a], noise[i, b] = float(z), 0.0
            want.append((i, a if score(a) + float(z) > score(b) else b))
    accepted, token, _ = bl.bitlogic_verify(
        x.to(DEV).expand(r, 2, c), torch.zeros((r, 1), dtype=torch.int32, device=DEV),
        torch.zeros(c, device=DEV).expand(r, 1, c), torch.full((r, 1), 0.9999999, device=DEV),
        noise, temperature=t_of.to(DEV))
    assert not accepted.any()
    assert token.cpu()[[w[0] for w in want]].tolist() == [w[1] for w in want]


def test_given_outputs_count_as_changed():
    case = Case(_rng(17), 6, 2, 40)
    outs = dict(accepted=torch.zeros(6, dtype=torch.int32, device=DEV),
                token=torch.zeros(6, dtype=torch.int32, device=DEV),
                log_prob=torch.ones(6, device=DEV))
    before = {name: t._version for name, t in outs.items()}
    case.check(case.run(**outs))
    assert all(t._version > before[name] for name, t in outs.items())


@pytest.mark.parametrize("near", [0.3, 2.0])
@pytest.mark.parametrize("r,d,c", [(420, 3, 1500), (500, 2, 2048), (850, 2, 4001), (850, 2, 4096)])
def test_many_requests_a_wave_each(r, d, c, near):
    test_many_requests(r, d, c, near)


@pytest.mark.parametrize("c,r", [(1500, 420), (4000, 850)])
def test_numbers_next_to_a_border_a_wave_each(c, r):
    test_numbers_next_to_a_border(c, r)
