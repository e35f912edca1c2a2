"""Dropout, adapters beside a quantized head, distillation, sampling and verification as they
are used together, and the example that does so."""
import os
import sys

import numpy as np
import pytest
import torch

import adapter_oracle
import draft_oracle
import logit_oracle
from paper_2602_07400_amd import bitlogic as bl

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))

pytestmark = pytest.mark.gpu

E = 2.0 ** -24                                            # half a step of float32


def test_example_runs():
    import adapt_head
    losses, (down, up), accepted, token, log_prob = adapt_head.run(samples=2003, steps=3)
    assert len(losses) == 3 and np.isfinite(losses).all()
    for g in (down, up):
        assert bool(torch.isfinite(g).all()) and bool((g != 0).any(2).any(1).all())
    assert accepted.shape == token.shape == log_prob.shape == (500,)
    assert bool(((accepted >= 0) & (accepted <= 3)).all())
    assert bool(((token >= 0) & (token < 10)).all())
    assert bool((log_prob <= 0).all()) and bool(torch.isfinite(log_prob).all())


@pytest.mark.parametrize("n,c,rank,groups,p", [(1, 10, 4, 3, 0.25), (300, 10, 4, 5, 0.1),
                                               (777, 100, 8, 24, 0.5)])
def test_gradients_of_the_run(n, c, rank, groups, p):
    """counts -> dropout -> adapters beside int32 logits -> distillation -> gradients, against
    the formulas in 64 bits."""
    rng = np.random.default_rng(n)
    counts = rng.integers(0, 40, (n, c)).astype(np.int32)
    base = rng.integers(-3000, 3000, (n, c)).astype(np.int32)
    ids = rng.integers(-1, groups, n).astype(np.int32)
    down = rng.normal(0, 0.2, (groups, rank, c)).astype(np.float32)
    up = rng.normal(0, 0.1, (groups, c, rank)).astype(np.float32)
    scales = rng.uniform(0.5, 1.5, groups).astype(np.float32)
    teacher = rng.integers(0, 40, (n, c)).astype(np.int32)
    base_scale, t, k = 0.0078125, 4.0, 4
    dev = lambda a: torch.from_numpy(a).cuda()            # noqa: E731
    values, classes, log_norm = bl.bitlogic_top_logits(dev(teacher), k, t)

    d, u = dev(down).requires_grad_(), dev(up).requires_grad_()
    dropped = bl.bitlogic_dropout(dev(counts), p, 5, offset=9)
    logits = bl.bitlogic_adapt(dropped, d, u, dev(ids), dev(scales), dev(base), base_scale)
    loss = bl.bitlogic_distill_loss(logits, values, classes, log_norm, t, t)
    got_down, got_up = torch.autograd.grad(loss.sum(), (d, u))

    x = draft_oracle.dropout(counts.astype(np.float64), p, 5, 9)
    assert (np.abs(dropped.cpu().numpy() - x) <= 2 * E * np.abs(x)).all()
    to64 = lambda a: a.astype(np.float64)                 # noqa: E731
    z, hidden, sizes = adapter_oracle.forward(x, to64(down), to64(up), ids, to64(scales),
                                              to64(base), base_scale)
    # of a logit: x rounded twice, products and sums of c and of rank terms, scale, base, sum
    off_z = (c + rank + 8) * E * sizes
    assert (np.abs(logits.detach().cpu().numpy() - z) <= off_z).all()

    grad, off = np.zeros((n, c)), np.zeros((n, c))
    for s in range(n):
        out = logit_oracle.distill(z[s], t, to64(values[s].cpu().numpy()),
                                   classes[s].cpu().numpy(), t, float(log_norm[s]))
        grad[s] = out[1]
        # logits off by d turn exponents by up to 2 d / t, each of the gradient's terms (each at
        # most 1 / t) by that share; an exponential's own error is below 4 |x| E, the list's and
        # the log-normalizer's among them, and a dozen roundings of sums are E each
        turn = 2 * off_z[s].max() / t
        size = 4 * (np.abs(z[s]).max() + np.abs(teacher[s]).max()) / t + c + 16
        off[s] = 4 * (turn + size * E) / t
    assert (np.abs(grad) <= 2 / t).all()
    _, (want_down, size_down), (want_up, size_up) = adapter_oracle.backward(
        grad, x, to64(down), to64(up), ids, to64(scales))
    _, (_, off_down), (_, off_up) = adapter_oracle.backward(
        off, np.abs(x), np.abs(to64(down)), np.abs(to64(up)), ids, to64(scales))
    rows = c + rank + n + 8                               # roundings of sums on the way
    assert (np.abs(got_down.cpu().numpy() - want_down) <=
            off_down + rows * E * (size_down + off_down)).all()
    assert (np.abs(got_up.cpu().numpy() - want_up) <=
            off_up + rows * E * (size_up + off_up)).all()
    assert (ids < 0).all() or float(got_up.abs().max()) > 0


def test_adapted_logits_are_drafted_and_verified():
    rng = np.random.default_rng(3)
    r, d, c, groups, rank, t = 60, 3, 20, 4, 4, 6.0
    n = r * (d + 1)
    dev = lambda a: torch.from_numpy(a).cuda()            # noqa: E731
    counts = rng.integers(0, 30, (n, c)).astype(np.int32)
    base = rng.integers(0, 3000, (n, c)).astype(np.int32)
    ids = rng.integers(-1, groups, n).astype(np.int32)
    down = rng.normal(0, 0.2, (groups, rank, c)).astype(np.float32)
    up = rng.normal(0, 0.2, (groups, c, rank)).astype(np.float32)
    target = rng.integers(0, 30, (r, d + 1, c)).astype(np.int32)
    gumbel = lambda *s: (-np.log(rng.exponential(size=s))).astype(np.float32)   # noqa: E731
    noise, own, uniform = gumbel(r, c), gumbel(n, c), rng.random((r, d)).astype(np.float32)
    logits, _ = bl.bitlogic_adapters(dev(counts), dev(down), dev(up), dev(ids), 1.0, dev(base),
                                     0.01)
    drafted = bl.bitlogic_sample(logits, dev(own), t)[0].view(r, d + 1)[:, :d].contiguous()
    drafter = logits.view(r, d + 1, c)[:, :d]             # strided from request to request
    accepted, token, log_prob = bl.bitlogic_verify(dev(target), drafted, drafter, dev(uniform),
                                                   dev(noise), temperature=t)
    y, classes = drafter.cpu().numpy().astype(np.float64), drafted.cpu().numpy()
    none = np.zeros((d + 1, c), bool)
    for s in range(r):
        want = draft_oracle.verify(target[s].astype(np.float64), none, classes[s], y[s],
                                   none[:d], uniform[s].astype(np.float64),
                                   noise[s].astype(np.float64), t, t)
        assert (int(accepted[s]), int(token[s])) == want[:2]
        # a log of a sum: within 1e-5 of the sum, the quotient and the result rounded to 32 bits
        assert abs(float(log_prob[s]) - want[2]) <= 1e-5 + 4 * E * (1 + abs(want[2]))


def test_run_in_a_graph():
    """The forward pass and the gradients of a step, captured once and replayed on new counts and
    offsets, with work of the program's own between replays."""
    rng = np.random.default_rng(7)
    n, c, groups, rank, t = 500, 10, 5, 4, 4.0
    ids = torch.from_numpy(rng.integers(0, groups, n).astype(np.int32)).cuda()
    base = torch.from_numpy(rng.integers(-900, 900, (n, c)).astype(np.int32)).cuda()
    scores = torch.from_numpy(rng.integers(0, 30, (n, c)).astype(np.int32)).cuda()
    down = torch.randn(groups, rank, c, device="cuda") * 0.1
    up = torch.randn(groups, c, rank, device="cuda") * 0.1
    values, classes, log_norm = bl.bitlogic_top_logits(scores, 4, t)
    counts, offset = scores.clone(), torch.zeros(1, dtype=torch.int64, device="cuda")
    plan = bl.bitlogic_group_rows(ids, groups)

    def step():
        x = bl.bitlogic_dropout(counts, 0.25, 11, offset=offset)
        z, hidden = bl.bitlogic_adapters(x, down, up, ids, 1.0, base, 0.01, plan,
                                         want_hidden=True)
        loss, grad = bl.bitlogic_distill(z, values, classes, log_norm, t, t)
        return loss, *bl.bitlogic_adapters_backward(grad, x, hidden, down, up, ids, 1.0, plan)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for i in range(4):
        counts.copy_(torch.from_numpy(rng.integers(0, 30, (n, c)).astype(np.int32)))
        offset.fill_(1000 * i)
        graph.replay()
        replayed = [v.clone() for v in captured]
        torch.cuda.synchronize()
        for a, b in zip(replayed, step()):                # the same kernels on the same inputs
            assert torch.equal(a, b)
