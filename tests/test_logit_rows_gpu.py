"""Top logits, distillation and sampling on rows of class scores against the 64-bit
oracle: every element type, class counts on both sides of each kernel layout's
limits, masks, ties, strides and alignments.

Tolerances.  Orders, classes, values and tokens are exact.  A sum of exponentials is
taken in 32 bits, at most about 130 terms a lane and ten levels across lanes, with
exponents rounded at 2^-24 of themselves: relative error below REL = 1e-5 and
2^-22 of the largest exponent M.  A log-probability's error is that, absolutely; the
loss is a mean of them under q; a gradient's is that share of the terms it is the
difference of, and its type's rounding."""
import numpy as np
import pytest
import torch

import logit_oracle as oracle
from paper_2602_07400_amd import bitlogic as bl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
REL = 1e-5
EPS = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
FLOATS = [torch.float32, torch.float16, torch.bfloat16]
TYPES = [torch.int32] + FLOATS
# both sides of the limits between layouts, of either element size
SIZES = [1, 2, 10, 16, 17, 37, 64, 65, 100, 128, 129, 500, 512, 513, 1000, 1024, 1025, 4097,
         8192, 8193, 32003, 32769, 50021, 65536, 65537, 131072, 131075]


def _rng(*key):
    return np.random.default_rng([5, *[int(k) for k in key]])


def _logits(rng, n, c, dtype, spread=3.0):
    if dtype == torch.int32:
        return torch.from_numpy(rng.integers(0, 641, (n, c)).astype(np.int32))
    return torch.from_numpy(rng.normal(0, spread, (n, c)).astype(np.float32)).to(dtype)


def _host(t):
    """(values in 64 bits, masked) of a tensor of logits."""
    x = t.detach().cpu()
    x = x.double().numpy() if x.dtype != torch.int32 else x.numpy().astype(np.float64)
    masked = np.isnan(x) | (x == (-2.0 ** 31 if t.dtype == torch.int32 else -np.inf))
    return x, masked


# ---------------------------------------------------------------- top logits

def _check_top(logits, k, temperature=1.0, **kw):
    values, indices, log_norm = bl.bitlogic_top_logits(logits, k, temperature, **kw)
    torch.cuda.synchronize()
    x, masked = _host(logits)
    cls, norm = oracle.top(x, masked, k, temperature)
    assert np.array_equal(indices.cpu().numpy(), cls)
    got = values.cpu()
    lowest = torch.tensor(-2 ** 31 if logits.dtype == torch.int32 else -np.inf,
                          dtype=logits.dtype)
    there = torch.from_numpy(cls.clip(0))
    want = torch.where(torch.from_numpy(cls >= 0), logits.cpu().gather(1, there), lowest)
    assert torch.equal(got, want)
    n = log_norm.cpu().numpy().astype(np.float64)
    fine = np.isfinite(norm)
    assert np.array_equal(n[~fine], norm[~fine])
    assert (np.abs(n - norm)[fine] <= REL + 2.0 ** -22 * np.abs(norm[fine])).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", SIZES)
def test_top_sizes(c, dtype):
    rng = _rng(1, c, TYPES.index(dtype))
    n = 37 if c <= 1024 else 5
    x = _logits(rng, n, c, dtype).to(DEV)
    for k in {1, min(c, 10), min(c, 257), min(c + 3, 1024)}:
        _check_top(x, k, 20.0 if dtype == torch.int32 else 0.7)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [10, 100, 300, 1000, 8000, 40001, 140000])
def test_top_masks_and_ties(c, dtype):
    rng = _rng(2, c, TYPES.index(dtype))
    x = _logits(rng, 9, c, dtype)
    low = torch.iinfo(dtype).min if dtype == torch.int32 else -np.inf
    x[0] = low                                            # nothing in the row
    x[1] = low
    x[1, c // 2] = 3                                      # one class
    x[2] = 7                                              # all equal
    x[3] = x[3] // 64 if dtype == torch.int32 else torch.round(x[3])   # many equal
    x[4, rng.integers(0, c, c)] = low
    if dtype != torch.int32:
        x[5, ::3] = np.nan
        x[6] = torch.finfo(dtype).min                     # a mask of the lowest value
        x[6, -1] = -torch.finfo(dtype).max / 2
        x[7, c // 3] = np.inf
        x[8] = torch.where(torch.arange(c) % 2 == 0, 0.0, -0.0)
    else:
        x[5] = 2 ** 31 - 1
        x[6, 0], x[6, -1] = 2 ** 31 - 1, -2 ** 31 + 1
        x[7] = -x[7]
        x[8] = 2 ** 30 + torch.arange(c, dtype=torch.int32) % 3        # above 2^24
    x = x.to(DEV)
    for k in (1, 5, min(c, 700), 1024):
        _check_top(x, k)


def test_top_strides_and_outputs():
    rng = _rng(3)
    for dtype in TYPES:
        wide = _logits(rng, 12, 3000, dtype).to(DEV)
        for view in (wide[:, 1:1000], wide[:, 7:2048], wide[::3, 3:103], wide[2:3, 5:2900],
                     wide[:1, 9:1200].expand(6, -1)):
            _check_top(view, 20)
    x = _logits(rng, 8, 500, torch.float32).to(DEV)
    v, i = torch.empty((8, 4), device=DEV), torch.empty((8, 4), dtype=torch.int32, device=DEV)
    rv, ri, norm = bl.bitlogic_top_logits(x, 4, values=v, indices=i, want_log_norm=False)
    assert rv is v and ri is i and norm is None
    assert torch.equal(v, torch.topk(x, 4).values)


def test_no_rows():
    x = torch.empty((0, 10), device=DEV)
    v, i, n = bl.bitlogic_top_logits(x, 3)
    assert v.shape == (0, 3) and i.shape == (0, 3) and n.shape == (0,)
    loss, grad = bl.bitlogic_distill(x, v, i, n)
    assert loss.shape == (0,) and grad.shape == (0, 10)
    token, log_prob = bl.bitlogic_sample(x, x)
    assert token.shape == (0,) and log_prob.shape == (0,)


# -------------------------------------------------------------- distillation

def _teacher(rng, n, c, k, dtype=torch.float32):
    idx = np.stack([rng.permutation(c)[:k] if k <= c else
                    np.concatenate([rng.permutation(c), np.full(k - c, -1)])
                    for _ in range(n)]).astype(np.int32)
    t = np.sort(rng.normal(3, 2, (n, k)))[:, ::-1].astype(np.float32)
    t = torch.from_numpy(t.copy())
    t = (t * 20).to(dtype) if dtype == torch.int32 else t.to(dtype)
    return t, torch.from_numpy(idx)


def _norm(t, idx, top_temperature, share):
    """A log-normalizer under which the list has `share` of the mass."""
    y = np.where(idx.numpy() >= 0, _host(t)[0], -np.inf) / top_temperature
    return torch.from_numpy((oracle.log_sum(y) - np.log(share)).astype(np.float32))


def _check_distill(z, t, idx, log_norm, temperature, top_temperature, weight, got):
    loss, grad = (v.cpu() if v is not None else None for v in got)
    x, masked = _host(z)
    x[masked & ~np.isnan(x)] = -np.inf                    # (the lowest int32 is a mask too)
    tv, iv = _host(t)[0], idx.cpu().numpy()
    for r in range(z.shape[0]):
        w = 1.0 if weight is None else float(weight[r])
        ln = None if log_norm is None else float(log_norm[r])
        want, g, p, q, q_rest, p_rest = oracle.distill(x[r], temperature, tv[r], iv[r],
                                                       top_temperature, ln)
        have = have_list = (iv[r] >= 0) & (iv[r] < z.shape[1])
        M = max(np.abs(x[r][np.isfinite(x[r])]).max(initial=0) / temperature,
                np.abs(tv[r][have]).max(initial=0) / top_temperature,
                abs(ln) if ln is not None and np.isfinite(ln) else 0)
        rel = 3 * REL + 2.0 ** -20 * M
        if loss is not None:
            if w == 0:
                assert float(loss[r]) == 0
            elif np.isfinite(want):
                assert abs(float(loss[r]) - w * want) <= abs(w) * rel * (1 + abs(want)), r
            else:
                assert str(float(loss[r])) == str(w * want), r
        if grad is not None:
            have = grad[r].double().numpy()
            if w == 0:
                assert (have == 0).all()
                continue
            g = w * g
            assert np.array_equal(np.isnan(have), np.isnan(g)), r
            fine = ~np.isnan(g)
            listed = np.zeros(len(p), bool)
            listed[iv[r][have_list]] = True
            rest = np.where(listed, -np.inf, x[r] / temperature)
            top = oracle.log_sum(rest)
            back = q_rest * np.exp(rest - top) if np.isfinite(top) else np.zeros(len(p))
            tol = (abs(w) / temperature * ((q.sum() + q_rest) * p + q + back) * rel
                   + EPS[z.dtype] * np.abs(g) + TINY[z.dtype])
            assert (np.abs(have - g)[fine] <= tol[fine]).all(), r


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("c", SIZES)
def test_distill_sizes(c, dtype):
    rng = _rng(4, c, TYPES.index(dtype))
    n = 19 if c <= 1024 else 4
    z = _logits(rng, n, c, dtype).to(DEV)
    for k in {1, min(c, 10), min(c, 130)}:
        t, idx = _teacher(rng, n, c, k, dtype)
        weight = torch.from_numpy(rng.uniform(0.2, 2, n).astype(np.float32))
        weight[1] = 0
        for rest in (False, True):
            if rest and k == c:
                continue
            ln = _norm(t, idx, 1.5, 0.8) if rest else None
            got = bl.bitlogic_distill(z, t.to(DEV), idx.to(DEV), None if ln is None else ln.to(DEV),
                                      2.0, 1.5, weight.to(DEV))
            torch.cuda.synchronize()
            _check_distill(z, t, idx, ln, 2.0, 1.5, weight, got)


@pytest.mark.parametrize("c", [10, 100, 700, 5000, 70001, 140000])
def test_distill_separate_calls_and_types(c):
    rng = _rng(5, c)
    z = _logits(rng, 6, c, torch.float32).to(DEV)
    for dtype in TYPES:
        t, idx = _teacher(rng, 6, c, 9, dtype)
        tt = 20.0 if dtype == torch.int32 else 1.0
        ln = _norm(t, idx, tt, 0.6)
        args = (z, t.to(DEV), idx.to(DEV), ln.to(DEV), 1.0, tt)
        loss, grad = bl.bitlogic_distill(*args)
        _check_distill(z, t, idx, ln, 1.0, tt, None, (loss, grad))
        one, none = bl.bitlogic_distill(*args, want_grad=False)
        assert none is None and torch.equal(one, loss)
        none, two = bl.bitlogic_distill(*args, want_loss=False)
        assert none is None and torch.equal(two, grad)
    # int32 scores of the student: the loss alone
    s = _logits(rng, 6, c, torch.int32).to(DEV)
    t, idx = _teacher(rng, 6, c, 9)
    loss, _ = bl.bitlogic_distill(s, t.to(DEV), idx.to(DEV), None, 16.0, want_grad=False)
    _check_distill(s, t, idx, None, 16.0, 1.0, None, (loss, None))


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("c", [12, 90, 600, 9000, 140000])
def test_distill_masks(c, rest):
    rng = _rng(6, c, rest)
    for dtype in FLOATS:
        z = _logits(rng, 11, c, dtype)
        t, idx = _teacher(rng, 11, c, 8, dtype)
        ln = _norm(t, idx, 1.0, 0.7) if rest else None
        idx[0] = -1                                       # an empty list
        idx[1, 3:] = -1
        idx[2, ::2] = c                                   # out of range: empty places
        z[3, 1::2] = -np.inf                              # masked classes, some listed
        z[4] = -np.inf                                    # no class at all
        z[5] = torch.finfo(dtype).min
        z[5, int(idx[5, 0])] = 1
        z[6, c // 2] = np.nan
        t[7, 4:] = -np.inf
        z[8] = -np.inf                                    # only the list has mass
        z[8, idx[8].long()] = 1
        z[9] = 0
        if rest:
            ln[10] -= 5                                   # a list of more than all the mass
        weight = torch.ones(11)
        got = bl.bitlogic_distill(z.to(DEV), t.to(DEV), idx.to(DEV),
                                  ln.to(DEV) if rest else None, 1.0, 1.0, weight.to(DEV))
        torch.cuda.synchronize()
        _check_distill(z.to(DEV), t, idx, ln, 1.0, 1.0, weight, got)


def test_distill_strides():
    rng = _rng(7)
    for dtype in FLOATS:
        wide = _logits(rng, 9, 2500, dtype).to(DEV)
        for z in (wide[:, 1:100], wide[:, 3:1500], wide[::2, 5:2406], wide[:1, 1:900].expand(4, -1)):
            n, c = z.shape
            t, idx = _teacher(rng, n, c, 12, dtype)
            room = torch.full((n, c + 9), 7.0, dtype=dtype, device=DEV)
            loss, grad = bl.bitlogic_distill(z, t.to(DEV), idx.to(DEV), temperature=0.8,
                                             grad=room[:, 5:c + 5])
            torch.cuda.synchronize()
            _check_distill(z, t, idx, None, 0.8, 1.0, None, (loss, grad))
            assert (room[:, :5] == 7).all() and (room[:, c + 5:] == 7).all()


def test_distill_autograd():
    rng = _rng(8)
    for c in (100, 3001):
        t, idx = _teacher(rng, 14, c, 20)
        ln = _norm(t, idx, 1.3, 0.9)
        z = _logits(rng, 14, c, torch.float32).to(DEV).requires_grad_()
        t, idx, ln = t.to(DEV), idx.to(DEV), ln.to(DEV)
        loss = bl.bitlogic_distill_loss(z, t, idx, ln, 1.1, 1.3)
        weight = torch.from_numpy(rng.uniform(-1, 2, 14).astype(np.float32)).to(DEV)
        (loss * weight).sum().backward()
        _, grad = bl.bitlogic_distill(z.detach(), t, idx, ln, 1.1, 1.3, weight)
        assert torch.equal(z.grad, grad)
        z.grad = None
        bl.bitlogic_distill_loss(z, t, idx, ln, 1.1, 1.3).mean().backward()
        _, grad = bl.bitlogic_distill(z.detach(), t, idx, ln, 1.1, 1.3,
                                      torch.full((14,), 1 / 14, device=DEV))
        assert torch.equal(z.grad, grad)
        # the loss does not differ from the functional form, and has no second derivative
        assert torch.equal(loss, bl.bitlogic_distill(z.detach(), t, idx, ln, 1.1, 1.3,
                                                     want_grad=False)[0])


@pytest.mark.parametrize("rest", [False, True])
def test_distill_gradient_against_differences(rest):
    """Central differences of the 64-bit loss along random directions.  h = 1e-4: the
    differences' own error is h^2 times a third derivative below 1 (1e-8) and 1e-12 of
    rounding, so the gradient's tolerance decides."""
    rng = _rng(9, rest)
    for c in (11, 150, 2000):
        z = _logits(rng, 3, c, torch.float32, 1.5)
        t, idx = _teacher(rng, 3, c, 6)
        ln = _norm(t, idx, 1.0, 0.75) if rest else None
        _, grad = bl.bitlogic_distill(z.to(DEV), t.to(DEV), idx.to(DEV),
                                      ln.to(DEV) if rest else None, 1.7)
        grad = grad.cpu().double().numpy()
        for r in range(3):
            of = lambda x: oracle.distill(x, 1.7, t[r].double().numpy(), idx[r].numpy(), 1.0,
                                          float(ln[r]) if rest else None)[0]
            for _ in range(4):
                d = rng.normal(size=c)
                d /= np.linalg.norm(d)
                x, h = z[r].double().numpy(), 1e-4
                diff = (of(x + h * d) - of(x - h * d)) / (2 * h)
                assert abs(diff - grad[r] @ d) <= 1e-7 + 6 * REL


# ------------------------------------------------------------------ sampling

def _gumbel(rng, n, c):
    return torch.from_numpy(rng.gumbel(size=(n, c)).astype(np.float32))


def _check_sample(logits, noise, temperature, k, top_p, min_p, got):
    token, log_prob = (v.cpu().numpy() for v in got)
    x, masked = _host(logits)
    g = noise.cpu().double().numpy()
    n = x.shape[0]
    of = lambda v, r: float(v[r]) if isinstance(v, torch.Tensor) else float(v)
    for r in range(n):
        args = (x[r], masked[r], g[r], np.float32(of(temperature, r)), int(of(k, r)),
                np.float32(of(top_p, r)), np.float32(of(min_p, r)))
        # a sum's rounding may decide which class is the last one of a top-p
        right = [oracle.sample(*args, slack) for slack in (0.0, REL, -REL)]
        same = [a for a in right if a[0] == token[r]]
        assert same, (r, int(token[r]), [int(a[0]) for a in right])
        want = np.array([a[1] for a in same], dtype=np.float64)
        if np.isfinite(want[0]):
            assert (np.abs(log_prob[r] - want) <= 2 * REL + 2.0 ** -22 * np.abs(want)).any(), r
        else:
            assert log_prob[r] == want[0]


FILTERS = [(0, 1.0, 0.0), (1, 1.0, 0.0), (5, 1.0, 0.0), (50, 0.9, 0.0), (0, 0.9, 0.0),
           (0, 0.3, 0.0), (0, 1.0, 0.1), (700, 0.99, 0.01), (2000, 1.0, 0.0), (0, 0.0, 0.0),
           (0, 0.999, 0.001), (3, 0.5, 0.9)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", SIZES)
def test_sample_sizes(c, dtype):
    rng = _rng(10, c, TYPES.index(dtype))
    n = 23 if c <= 1024 else 3
    x = _logits(rng, n, c, dtype).to(DEV)
    noise = _gumbel(rng, n, c).to(DEV)
    scale = 30.0 if dtype == torch.int32 else 1.0
    for k, p, m in FILTERS:
        got = bl.bitlogic_sample(x, noise, 0.8 * scale, k, p, m)
        torch.cuda.synchronize()
        _check_sample(x, noise, 0.8 * scale, k, p, m, got)
    token, log_prob = bl.bitlogic_sample(x, temperature=0)
    assert torch.equal(token.cpu().long(), torch.from_numpy(
        np.argmax(_host(x)[0], axis=1)))
    assert (log_prob == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [10, 100, 300, 1000, 8000, 40001, 140000])
def test_sample_masks_ties_and_row_parameters(c, dtype):
    rng = _rng(11, c, TYPES.index(dtype))
    n = 12
    x = _logits(rng, n, c, dtype)
    low = torch.iinfo(dtype).min if dtype == torch.int32 else -np.inf
    x[0] = low
    x[1] = low
    x[1, c // 2] = 3
    x[2] = 7                                              # all equal
    x[3] = x[3] // 64 if dtype == torch.int32 else torch.round(x[3])
    x[4, rng.integers(0, c, c)] = low
    if dtype != torch.int32:
        x[5, ::3] = np.nan
        x[6] = torch.finfo(dtype).min                     # all at the lowest value
        x[7, c // 3] = np.inf
        x[7, c // 2] = np.inf
        x[8] = torch.where(torch.arange(c) % 2 == 0, 0.0, -0.0)
        x[9, 1:] = torch.finfo(dtype).min
    else:
        x[5] = 2 ** 31 - 1
        x[6, 0] = -2 ** 31 + 1
    noise = _gumbel(rng, n, c)
    noise[10, ::2] = -np.inf
    noise[11] = np.nan
    x, noise = x.to(DEV), noise.to(DEV)
    scale = 30.0 if dtype == torch.int32 else 1.0
    for shift in range(4):
        every = [FILTERS[(r + 3 * shift) % len(FILTERS)] for r in range(n)]
        t = torch.from_numpy(rng.uniform(0.3, 2, n).astype(np.float32) * scale)
        t[shift::5] = 0 if shift % 2 else t[shift::5]
        k = torch.tensor([f[0] for f in every], dtype=torch.int32)
        p = torch.tensor([f[1] for f in every], dtype=torch.float32)
        m = torch.tensor([f[2] for f in every], dtype=torch.float32)
        got = bl.bitlogic_sample(x, noise, t.to(DEV), k.to(DEV), p.to(DEV), m.to(DEV))
        torch.cuda.synchronize()
        _check_sample(x, noise, t, k, p, m, got)


def test_sample_strides():
    rng = _rng(12)
    for dtype in TYPES:
        wide = _logits(rng, 9, 2500, dtype).to(DEV)
        g = _gumbel(rng, 9, 2600).to(DEV)
        for rows, cols, off in ((slice(None), slice(1, 100), 3), (slice(None), slice(3, 1500), 1),
                                (slice(0, 9, 2), slice(5, 2406), 7)):
            x = wide[rows, cols]
            noise = g[:x.shape[0], off:off + x.shape[1]]
            t = 25.0 if dtype == torch.int32 else 0.9
            got = bl.bitlogic_sample(x, noise, t, 40, 0.95, 0.0)
            torch.cuda.synchronize()
            _check_sample(x, noise, t, 40, 0.95, 0.0, got)


def test_sample_frequencies():
    """Draws follow the filtered softmax: over 2^16 rows each class's count is within
    6 standard deviations of its expectation."""
    n, c = 1 << 16, 12
    logits = torch.linspace(0, 3, c, device=DEV).expand(n, -1)
    gen = torch.Generator(DEV).manual_seed(3)
    noise = -torch.empty((n, c), device=DEV).exponential_(generator=gen).log()
    token, log_prob = bl.bitlogic_sample(logits, noise, 1.5, 8, 0.9)
    _, _, kept = oracle.sample(np.linspace(0, 3, c).astype(np.float32).astype(np.float64),
                               np.zeros(c, bool), np.zeros(c), 1.5, 8, np.float32(0.9), 0.0)
    p = np.zeros(c)
    p[kept] = np.exp(np.linspace(0, 3, c)[kept] / 1.5)
    p /= p.sum()
    count = np.bincount(token.cpu().numpy(), minlength=c)
    assert (np.abs(count - n * p) <= 6 * np.sqrt(n * p * (1 - p)) + 1e-9).all()
    assert np.allclose(np.exp(log_prob.cpu().numpy()), p[token.cpu().numpy()], rtol=3 * REL)


# ------------------------------------------------------------ many short rows

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [1, 2, 10, 37, 63, 64, 65, 100, 127, 128])
def test_many_short_rows(c, dtype):
    """From 16384 rows on a lane takes a row: masks, ties, empty lists and strides among
    17003 rows, of which the oracle checks the first 150 and the last 60."""
    rng = _rng(16, c, TYPES.index(dtype))
    n = 17003
    wide = _logits(rng, n, c + 3, dtype)
    low = torch.iinfo(dtype).min if dtype == torch.int32 else -np.inf
    wide[::7, :] = torch.round(wide[::7, :].float()).to(dtype)
    wide[3, :] = low
    wide[4, 1:] = low
    wide[5, rng.integers(0, c, c)] = low
    wide[6] = 7
    if dtype != torch.int32:
        wide[8, ::2] = np.nan
        wide[9] = torch.finfo(dtype).min
        wide[10, :] = torch.where(torch.arange(c + 3) % 2 == 0, 0.0, -0.0)
    wide = wide.to(DEV)
    some = np.r_[0:150, n - 60:n]
    for x in (wide[:, 1:c + 1], wide[:, :c].contiguous()):
        for k in sorted({1, min(c, 4), 7, 12}):
            v, i, norm = bl.bitlogic_top_logits(x, k, 1.5)
            few = bl.bitlogic_top_logits(x[some], k, 1.5)
            assert torch.equal(i[some], few[1]) and torch.equal(v[some], few[0])
            d = (norm[some] - few[2]).abs()
            assert ((d <= 2 * REL + 2.0 ** -21 * few[2].abs()) | (norm[some] == few[2])).all()
            _check_top(x[some], k, 1.5)
        k = min(c, 9)
        t, idx = _teacher(rng, n, c, k, dtype)
        idx[20] = -1
        idx[21, 1:] = c
        tt = 20.0 if dtype == torch.int32 else 1.0
        weight = torch.from_numpy(rng.uniform(0.2, 2, n).astype(np.float32))
        weight[::11] = 0
        for rest in (False, True):
            if rest and k == c:
                continue
            ln = _norm(t, idx, tt, 0.8) if rest else None
            if rest:
                ln[20] = 0.0
            loss, grad = bl.bitlogic_distill(
                x, t.to(DEV), idx.to(DEV), None if ln is None else ln.to(DEV), 2.0, tt,
                weight.to(DEV), want_grad=dtype != torch.int32)
            torch.cuda.synchronize()
            _check_distill(x[some], t[some], idx[some], None if ln is None else ln[some], 2.0, tt,
                           weight[some], (loss[some], None if grad is None else grad[some]))


# ------------------------------------------------ addresses, streams, graphs

def test_offsets_past_32_bits():
    """Rows 2^30 elements apart: byte offsets of 8 and 12 GB."""
    rng = _rng(13)
    c, far = 3001, 1 << 30
    logits = torch.empty(2 * far + c, dtype=torch.float32, device=DEV).as_strided((3, c), (far, 1))
    grad = torch.empty(2 * far + c, dtype=torch.float32, device=DEV).as_strided((3, c), (far, 1))
    x = _logits(rng, 3, c, torch.float32).to(DEV)
    logits.copy_(x)
    for a, b in zip(bl.bitlogic_top_logits(logits, 30), bl.bitlogic_top_logits(x, 30)):
        assert torch.equal(a, b)
    t, idx = (v.to(DEV) for v in _teacher(rng, 3, c, 9))
    loss, _ = bl.bitlogic_distill(logits, t, idx, grad=grad)
    want, g = bl.bitlogic_distill(x, t, idx)
    assert torch.equal(loss, want) and torch.equal(grad, g)
    noise = _gumbel(rng, 3, c).to(DEV)
    grad.copy_(noise)
    for a, b in zip(bl.bitlogic_sample(logits, grad, 0.9, 20, 0.9),
                    bl.bitlogic_sample(x, noise, 0.9, 20, 0.9)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("c", [100, 40001])
def test_runs_agree_on_any_stream(c):
    rng = _rng(14, c)
    x = _logits(rng, 40, c, torch.bfloat16).to(DEV)
    noise = _gumbel(rng, 40, c).to(DEV)
    t, idx = (v.to(DEV) for v in _teacher(rng, 40, c, 30, torch.bfloat16))

    def everything(stream=None):
        return (*bl.bitlogic_top_logits(x, 50, stream=stream),
                *bl.bitlogic_distill(x, t, idx, stream=stream),
                *bl.bitlogic_sample(x, noise, 0.9, 0, 0.95, stream=stream))

    first = everything()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for got in (everything(), everything(side), everything(side.cuda_stream)):
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_graph_replays():
    rng = _rng(15)
    c = 3001
    x = _logits(rng, 8, c, torch.float16).to(DEV)
    noise = _gumbel(rng, 8, c).to(DEV)

    def step():
        v, i, n = bl.bitlogic_top_logits(x, 16, 1.2)
        loss, grad = bl.bitlogic_distill(x, v, i, n, 1.0, 1.2)
        token, log_prob = bl.bitlogic_sample(x, noise, 0.9, 30, 0.9)
        return v, i, n, loss, grad, token, log_prob

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for again in range(4):
        x.copy_(_logits(rng, 8, c, torch.float16))
        noise.copy_(_gumbel(rng, 8, c))
        graph.replay()
        torch.cuda.synchronize()
        kept = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(kept, step())), again
