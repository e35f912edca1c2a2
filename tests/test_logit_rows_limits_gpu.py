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


# ---------------------------------------------- rows of millions of classes

def _levels(rng, c, low, dtype):
    """One row of c classes, the second half (shuffled) `low` below the others."""
    x = torch.zeros(c, dtype=dtype)
    x[torch.from_numpy(rng.permutation(c)[c // 2:])] = low
    return x[None]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [1 << 20, (1 << 22) + 5, (1 << 24) + 3])
def test_sums_over_millions_of_classes(c, dtype):
    rng = _rng(22, c)
    x = torch.full((1, c), -1.2, dtype=dtype)
    x[0, c // 3] = 0
    w = np.exp(float(x[0, 0]))
    total = 1 + (c - 1) * w
    v, i, norm = bl.bitlogic_top_logits(x.to(DEV), 3)
    assert i.tolist() == [[c // 3, 0, 1]]
    assert abs(float(norm) - np.log(total)) <= REL + 2.0 ** -22 * np.log(total)
    noise = _gumbel(rng, 1, c)
    for min_p in (0.0, 0.2):                              # (every class is kept)
        token, log_prob = bl.bitlogic_sample(x.to(DEV), noise.to(DEV), 1.0, min_p=min_p)
        at = int(token)
        score = (x.float() + noise)[0]
        assert float(score[at]) == float(score.max())
        want = float(x[0, at]) - np.log(total)
        assert abs(float(log_prob) - want) <= 2 * REL + 2.0 ** -22 * abs(want)
    # two classes of a teacher's, the rest of 30%
    t, idx = torch.tensor([[1.0, 0.5]]), torch.tensor([[c // 3, 7]], dtype=torch.int32)
    ln = _norm(t, idx, 1.0, 0.7)
    loss, grad = bl.bitlogic_distill(x.to(DEV), t.to(DEV), idx.to(DEV), ln.to(DEV))
    q = np.exp(t.double().numpy()[0] - float(ln))
    p, p_rest, q_rest = np.array([1, w]) / total, (c - 2) * w / total, 1 - q.sum()
    want = (q * np.log(q / p)).sum() + q_rest * np.log(q_rest / p_rest)
    rel = 3 * REL + 2.0 ** -20 * 2
    assert abs(float(loss) - want) <= rel * (1 + abs(want))
    g = grad.cpu().double()[0]
    out = (1 - q_rest / p_rest) * w / total               # of each class outside the list
    tol = (1 + q_rest / p_rest) * w / total * rel + EPS[dtype] * abs(out) + TINY[dtype]
    rest = torch.ones(c, dtype=torch.bool)
    rest[[c // 3, 7]] = False
    assert float((g[rest] - out).abs().max()) <= tol
    assert (np.abs(g[~rest].flip(0).numpy() - (p - q)) <= (p + q) * rel + EPS[dtype]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("c", [1 << 17, 1 << 20, (1 << 22) + 5, (1 << 24) + 3])
def test_top_p_boundary_over_millions_of_classes(c, dtype):
    """Two levels, and a nucleus that ends among the lower ones: the kept mass is the
    target's to REL, whatever a class's share of it."""
    rng = _rng(23, c)
    x = _levels(rng, c, -0.2, dtype)
    noise = _gumbel(rng, 1, c)
    low = np.nonzero(x[0].float().numpy() < 0)[0]
    w, n = np.exp(float(x.min())), c - len(low)
    score = (x.float() + noise)[0].numpy()
    for top_p in (0.6, 0.9, 0.999):
        token, log_prob = bl.bitlogic_sample(x.to(DEV), noise.to(DEV), 1.0, top_p=top_p)
        total = n + len(low) * w
        need = float(np.float32(top_p)) * total - n
        assert need > 0
        slack = REL * total / w + 1
        kept = np.ones(c, bool)
        few, many = (int(np.clip(np.ceil(need / w) + s, 0, len(low))) for s in (-slack, slack))
        kept[low[few:]] = False
        best = score[kept].max()
        kept[low[few:many]] = True
        assert best <= score[int(token)] <= score[kept].max()
        want = float(x[0, int(token)]) - np.log(n + np.ceil(need / w) * w)
        assert abs(float(log_prob) - want) <= 3 * REL + 2.0 ** -22 * abs(want)


# ------------------------------------------------------------------- repeats

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [3000, 20000, 131072])
def test_sample_repeats_bit_for_bit(c, dtype):
    """Kept sets whose classes reach LDS in whatever order the waves get there: the
    log-probability's bits do not depend on it."""
    rng = _rng(24, c, TYPES.index(dtype))
    n = 64
    scale = 30.0 if dtype == torch.int32 else 1.0
    x = _logits(rng, n, c, torch.float32, 2.0 * scale).round() if dtype == torch.int32 \
        else _logits(rng, n, c, torch.float32, 2.0)
    x = x.to(dtype).to(DEV)
    noise = _gumbel(rng, n, c).to(DEV)
    for k, p, m in ((0, 1.0, 0.02), (0, 1.0, 0.002), (0, 0.95, 0.01), (2500, 1.0, 0.01),
                    (2500, 0.9, 0.0), (0, 0.9, 0.0)):
        first = bl.bitlogic_sample(x, noise, scale, k, p, m)
        for _ in range(12):
            again = bl.bitlogic_sample(x, noise, scale, k, p, m)
            torch.cuda.synchronize()
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]), (k, p, m)


# -------------------------------------------------------- scores past 2^24

@pytest.mark.parametrize("c", [12, 100, 700, 5000, 40001, 140000])
def test_scores_that_differ_below_their_float_rounding(c):
    """Int32 scores of 2^30 and more, a few units apart: what depends on differences alone
    is that of the scores less their maximum, which float holds exactly."""
    rng = _rng(25, c)
    n = 6
    near = torch.from_numpy(rng.integers(-40, 1, (n, c)).astype(np.int32))
    near[:, 0] = 0
    near[0, 1] = near[1, 2] = -2 ** 31                    # masked
    high = torch.where(near > -2 ** 31, near + 2 ** 30 + 7, near)
    noise = _gumbel(rng, n, c).to(DEV)
    for k, p, m in ((0, 1.0, 0.0), (5, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.05), (700, 0.99, 0.01),
                    (2000, 0.9, 0.0)):
        a = bl.bitlogic_sample(near.to(DEV), noise, 6.0, k, p, m)
        b = bl.bitlogic_sample(high.to(DEV), noise, 6.0, k, p, m)
        torch.cuda.synchronize()
        _check_sample(near, noise, 6.0, k, p, m, a)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), (k, p, m)
    # the student's scores, and the teacher's (its list's own normalizer)
    t, idx, _ = bl.bitlogic_top_logits(high.to(DEV), 9, 6.0)
    for i in range(9):
        assert (idx[:, i] >= 0).all()
    shifted = (t.cpu() - (2 ** 30 + 7)).to(DEV)
    for z in (near, high):
        for v in (shifted, t):
            loss, _ = bl.bitlogic_distill(z.to(DEV), v, idx, None, 6.0, 6.0, want_grad=False)
            _check_distill(near, shifted.cpu(), idx.cpu(), None, 6.0, 6.0, None, (loss, None))


def test_many_short_rows_of_scores_past_2_24():
    rng = _rng(26)
    n, c = 17003, 37
    near = torch.from_numpy(rng.integers(-40, 1, (n, c)).astype(np.int32))
    near[:, 5] = 0
    near[3, 1] = -2 ** 31
    high = torch.where(near > -2 ** 31, near + 2 ** 30 + 7, near).to(DEV)
    near = near.to(DEV)
    t, idx, norm = bl.bitlogic_top_logits(high, 9, 4096.0)
    shifted, same, base = bl.bitlogic_top_logits(near, 9, 4096.0)
    assert torch.equal(idx, same) and torch.equal(t - (2 ** 30 + 7), shifted)
    far = base.double() + (2.0 ** 30 + 7) / 4096
    assert bool(((norm - far).abs() <= REL + 2.0 ** -23 * far).all())
    want, _ = bl.bitlogic_distill(near, shifted, idx, None, 6.0, 6.0, want_grad=False)
    some = np.r_[0:60, n - 30:n]
    _check_distill(near[some].cpu(), shifted[some].cpu(), idx[some].cpu(), None, 6.0, 6.0, None,
                   (want[some], None))
    for z in (near, high):
        for v in (shifted, t):
            loss, _ = bl.bitlogic_distill(z, v, idx, None, 6.0, 6.0, want_grad=False)
            assert bool(((loss - want).abs() <= 3 * REL * (1 + want.abs())).all())


# ---------------------------------------------- ends of the parameters' ranges

@pytest.mark.parametrize("c", [12, 100, 700, 5000, 140000])
def test_sample_min_p_above_one_keeps_the_first_class(c):
    rng = _rng(27, c)
    x = torch.zeros((3, c))
    x[1, c // 2:] = -1.0
    x[2, ::2] = 3.0
    noise = _gumbel(rng, 3, c)
    m = torch.tensor([1.5, 2.0, 100.0])
    for k, p in ((0, 1.0), (5, 1.0), (0, 0.9), (2000, 0.9)):
        got = bl.bitlogic_sample(x.to(DEV), noise.to(DEV), 1.0, k, p, m.to(DEV))
        torch.cuda.synchronize()
        _check_sample(x, noise, 1.0, k, p, m, got)
        assert got[0].tolist() == [0, 0, 0] and (got[1] == 0).all()


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("c", [12, 100, 700, 5000, 140000])
def test_sample_infinite_logits_at_any_temperature(c, dtype):
    """Beside a logit of +inf no finite one has mass: not the type's largest either, nor
    at a temperature of 1e38."""
    rng = _rng(28, c, FLOATS.index(dtype))
    x = _logits(rng, 4, c, dtype)
    x[0, c // 3] = np.inf
    x[1, c // 3] = np.inf
    x[1, c // 2] = torch.finfo(dtype).max
    x[2] = torch.finfo(dtype).max
    x[2, [1, c - 2]] = np.inf
    noise = _gumbel(rng, 4, c)
    for t in (1.0, 1e38):
        for k, p, m in ((0, 1.0, 0.0), (5, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.05),
                        (700, 0.99, 0.01), (5, 0.9, 0.0)):
            got = bl.bitlogic_sample(x.to(DEV), noise.to(DEV), t, k, p, m)
            torch.cuda.synchronize()
            _check_sample(x, noise, t, k, p, m, got)


@pytest.mark.parametrize("n", [3, 17003])
@pytest.mark.parametrize("c", [12, 100, 700, 5000, 140000])
def test_temperatures_below_the_normal_numbers(c, n):
    """A temperature below 2^-126, whose reciprocal may be no float, counts as 2^-126:
    the largest logits share all the mass."""
    if n > 3 and c > 128:
        pytest.skip("many short rows only")
    rng = _rng(29, c, n)
    x = _logits(rng, n, c, torch.float32)
    x = x - x.max(1, keepdim=True).values
    x[:, [1, c // 2]] = 0                                 # the largest, equal
    noise = _gumbel(rng, n, c).to(DEV)
    x = x.to(DEV)
    top = (x == 0)
    first, count = top.int().argmax(1).int(), top.sum(1)
    t, idx = torch.zeros((n, 2), device=DEV), torch.zeros((n, 2), dtype=torch.int32, device=DEV)
    idx[:, 0], idx[:, 1] = 1, c // 2
    for temperature in (1e-39, 2.0 ** -126):
        v, i, norm = bl.bitlogic_top_logits(x, 3, temperature)
        assert torch.equal(i[:, 0], first)
        assert bool(((norm - count.log()).abs() <= REL).all())
        loss, grad = bl.bitlogic_distill(x, t, idx, None, temperature, 1.0)
        assert bool(((loss - (count.log() - np.log(2))).abs() <= 3 * REL).all())
        assert bool((grad[~top] == 0).all())
        loss, _ = bl.bitlogic_distill(x, t, idx, None, 1.0, temperature, want_grad=False)
        assert bool(torch.isfinite(loss).all())
        same, _ = bl.bitlogic_distill(x, t, idx, None, 1.0, 1.0, want_grad=False)
        assert torch.equal(loss, same)                    # (equal entries at any temperature)
        if n > 3:
            continue
        for p in (1.0, 0.9):
            for given in (temperature, torch.full((n,), temperature, device=DEV)):
                token, log_prob = bl.bitlogic_sample(x, noise, given, 0, p)
                kept = torch.ceil(count * float(np.float32(p)))
                assert bool(top.gather(1, token.long()[:, None]).all())
                assert bool(((log_prob + kept.log()).abs() <= 2 * REL).all())


def test_distill_at_the_largest_temperatures():
    """Logits of the size of a temperature of 1e38: differences of the order of one."""
    rng = _rng(30)
    for c in (12, 700, 5000):
        x = torch.from_numpy(rng.uniform(-1.4e38, 1.4e38, (4, c)).astype(np.float32))
        t, idx = _teacher(rng, 4, c, 5)
        ln = _norm(t, idx, 1.0, 0.7)
        got = bl.bitlogic_distill(x.to(DEV), t.to(DEV), idx.to(DEV), ln.to(DEV), 1e38)
        torch.cuda.synchronize()
        _check_distill(x, t, idx, ln, 1e38, 1.0, None, (got[0], None))


# ----------------------------------------------------- more rows than one launch

def _windows(n, c, rng):
    """n rows of c classes that start one element apart."""
    block = torch.from_numpy(rng.normal(0, 3, 1 << 20).astype(np.float32)).to(DEV)
    flat = block.repeat((n + c) // (1 << 20) + 1)
    flat.add_(torch.arange(flat.numel(), device=DEV) % 8191, alpha=2.0 ** -10)
    return flat[:n + c].as_strided((n, c), (1, 1))


def test_rows_past_one_launch():
    """2^24 rows of a block of 256 lanes are 2^32 lanes, which no launch has."""
    rng = _rng(33)
    n, c = (1 << 24) + 3, 1025
    x, noise = _windows(n, c, rng), _windows(n, c, rng)
    some = torch.tensor([0, 1, 77, n // 2, *range(n - 262, n)], device=DEV)
    for a, b in zip(bl.bitlogic_top_logits(x, 2), bl.bitlogic_top_logits(x[some], 2)):
        assert torch.equal(a[some], b)
    t = torch.rand((n, 1), device=DEV)
    idx = (torch.arange(n, device=DEV, dtype=torch.int32) % c)[:, None]
    norm, weight = t[:, 0] + 0.25, 1 + t[:, 0]
    loss, _ = bl.bitlogic_distill(x, t, idx, norm, 1.1, row_weight=weight, want_grad=False)
    few, _ = bl.bitlogic_distill(x[some], t[some], idx[some], norm[some], 1.1,
                                 row_weight=weight[some], want_grad=False)
    assert torch.equal(loss[some], few)
    k = torch.arange(n, device=DEV, dtype=torch.int32) % 60
    for each in ((0.5 + t[:, 0], k, 0.3 + 0.7 * t[:, 0], 0.1 * t[:, 0]), (0.9, 0, 1.0, 0.0)):
        of = [v[some] if torch.is_tensor(v) else v for v in each]
        token, log_prob = bl.bitlogic_sample(x, noise, *each)
        few = bl.bitlogic_sample(x[some], noise[some], *of)
        assert torch.equal(token[some], few[0]) and torch.equal(log_prob[some], few[1])


def test_short_rows_past_one_launch():
    """2^30 rows of four lanes each."""
    n = (1 << 30) + 70
    x = _windows(n, 2, _rng(34))
    t = torch.ones((n, 1), device=DEV)
    idx = torch.zeros((n, 1), dtype=torch.int32, device=DEV)
    t[n - 64:] = 2
    idx[n - 70:n - 10] = 1
    norm = t[:, 0] + 0.25
    loss, _ = bl.bitlogic_distill(x, t, idx, norm, 1.1, want_grad=False)
    some = torch.arange(n - 20000, n, device=DEV)
    few, _ = bl.bitlogic_distill(x[some], t[some], idx[some], norm[some], 1.1, want_grad=False)
    assert torch.equal(loss[some], few) and torch.equal(
        loss[:20000], bl.bitlogic_distill(x[:20000], t[:20000], idx[:20000], norm[:20000], 1.1,
                                          want_grad=False)[0])


# ------------------------------------------------------------------ long lists

@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("c", [10, 16, 17, 64, 65, 128, 129, 512, 513, 1024, 1025, 8193, 70001,
                               140000])
def test_distill_long_lists(c, dtype, rest):
    """Lists of up to 1024 entries, some longer than the row (places left empty)."""
    rng = _rng(31, c, FLOATS.index(dtype), rest)
    n = 9 if c <= 1024 else 3
    z = _logits(rng, n, c, dtype).to(DEV)
    for k in (257, 820, 1024):
        t, idx = _teacher(rng, n, c, k, dtype)
        ln = _norm(t, idx, 1.5, 0.8) if rest and k < c else None
        weight = torch.from_numpy(rng.uniform(0.2, 2, n).astype(np.float32))
        args = (z, t.to(DEV), idx.to(DEV), None if ln is None else ln.to(DEV), 2.0, 1.5,
                weight.to(DEV))
        got = bl.bitlogic_distill(*args)
        alone, _ = bl.bitlogic_distill(*args, want_grad=False)
        torch.cuda.synchronize()
        _check_distill(z, t, idx, ln, 2.0, 1.5, weight, got)
        assert torch.equal(alone, got[0])


@pytest.mark.parametrize("dtype", FLOATS)
def test_distill_autograd_in_every_type(dtype):
    rng = _rng(32, FLOATS.index(dtype))
    for c in (10, 100, 3001, 70001):
        t, idx = _teacher(rng, 5, c, 7, dtype)
        ln = _norm(t, idx, 1.3, 0.9).to(DEV)
        z = _logits(rng, 5, c, dtype).to(DEV).requires_grad_()
        loss = bl.bitlogic_distill_loss(z, t.to(DEV), idx.to(DEV), ln, 1.1, 1.3)
        weight = torch.from_numpy(rng.uniform(-1, 2, 5).astype(np.float32)).to(DEV)
        (loss * weight).sum().backward()
        want, grad = bl.bitlogic_distill(z.detach(), t.to(DEV), idx.to(DEV), ln, 1.1, 1.3, weight)
        assert z.grad.dtype == dtype and torch.equal(z.grad, grad)
        assert torch.equal(loss.detach() * weight, want) or bool(
            ((loss.detach() * weight - want).abs() <= 2.0 ** -22 * want.abs()).all())
        _check_distill(z.detach(), t, idx, ln.cpu(), 1.1, 1.3, weight, (None, grad))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("c", [10, 100, 127, 128])
def test_top_lists_by_lanes(c, dtype):
    """Enough rows that a lane takes one, 256 a class, and one row less: the same lists."""
    rng = _rng(35, c, TYPES.index(dtype))
    n = 256 * c
    x = _logits(rng, n, c, dtype)
    low = torch.iinfo(dtype).min if dtype == torch.int32 else -np.inf
    x[3] = low
    x[4, 1:] = low
    x[5] = 7
    x[n - 1, ::2] = low
    x = x.to(DEV)
    some = np.r_[0:60, n - 30:n]
    for k in (1, 5, 8, 12):
        v, i, norm = bl.bitlogic_top_logits(x, k, 1.5)
        few = bl.bitlogic_top_logits(x[1:], k, 1.5)
        assert torch.equal(v[1:], few[0]) and torch.equal(i[1:], few[1])
        d = (norm[1:] - few[2]).abs()
        assert bool(((d <= 2 * REL + 2.0 ** -21 * few[2].abs()) | (norm[1:] == few[2])).all())
        _check_top(x[some], k, 1.5)


@pytest.mark.parametrize("top_type", TYPES)
@pytest.mark.parametrize("c,n", [(12, 5), (100, 17003), (700, 5), (9000, 5)])
def test_distill_lists_of_masked_values(c, n, top_type):
    """A list whose values are all masked is an empty one; masked values beside others have
    no mass."""
    rng = _rng(36, c, TYPES.index(top_type))
    z = _logits(rng, n, c, torch.float32).to(DEV)
    t, idx = _teacher(rng, n, c, 6, top_type)
    low = torch.iinfo(torch.int32).min if top_type == torch.int32 else -np.inf
    t[0] = low
    t[1, 2:] = low
    tt = 20.0 if top_type == torch.int32 else 1.0
    loss, grad = bl.bitlogic_distill(z, t.to(DEV), idx.to(DEV), None, 1.5, tt)
    assert float(loss[0]) == 0 and bool((grad[0] == 0).all())
    empty = idx.clone()
    empty[1, 2:] = -1
    want = bl.bitlogic_distill(z, t.to(DEV), empty.to(DEV), None, 1.5, tt)
    assert abs(float(loss[1] - want[0][1])) <= 3 * REL * (1 + abs(float(want[0][1])))
    # (the gradient of a class that is listed with no mass is p, as of one that is not)
    assert bool(((grad[1] - want[1][1]).abs() <= 3 * REL * want[1][1].abs() + 1e-37).all())
    _check_distill(z[2:5].cpu(), t[2:5], idx[2:5], None, 1.5, tt, None, (loss[2:5], grad[2:5]))


def test_sample_top_k_past_32_bits():
    rng = _rng(37)
    x, noise = _logits(rng, 4, 50, torch.float32).to(DEV), _gumbel(rng, 4, 50).to(DEV)
    want = bl.bitlogic_sample(x, noise, 2.0)
    for k in (51, 2 ** 31, 2 ** 32 + 1):
        got = bl.bitlogic_sample(x, noise, 2.0, k)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(Exception, match="top_k"):
        bl.bitlogic_sample(x, noise, 2.0, -1)
