"""Adapt the quantized head of a small LUT network to several sources of inputs, and let the
adapted network draft labels for a wider one.

The small network and its int8 head are deployed as they are.  Each source of inputs has a
low-rank adapter beside the head, fitted against a wider network's top scores
(bitlogic_top_logits, bitlogic_distill_loss) with dropout on the counts (bitlogic_dropout,
bitlogic_adapt); rows of all sources go through one call, grouped once (bitlogic_group_rows).
Then the adapted network draws labels for a few inputs of each request (bitlogic_sample), and
the wide network keeps those that stand by its own probabilities and draws the next label
itself (bitlogic_verify): labels as if it had drawn all of them.

    python examples/adapt_head.py [--samples N] [--steps K]

Needs the built library and a GPU; networks and pixels are seeded synthetic ones.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2602_07400_amd import bitlogic as bl                      # noqa: E402
from paper_2602_07400_amd import workloads as wk                     # noqa: E402


def network(rng, n_features, widths, k):
    """Thresholds and layers of a network with one threshold a feature."""
    w_in, layers = n_features, []
    for w in widths:
        layers.append((wk.draw_connectivity(rng, w, k, w_in), wk.draw_tables(rng, w, k)))
        w_in = w
    return np.full((n_features, 1), 127, np.uint8), layers


def run(samples=8192, steps=60, sources=5, rank=4, drafts=3, n_features=784, n_classes=10,
        temperature=8.0, drop=0.1, seed=0, device="cuda"):
    """Returns the losses of the fit, the last gradients of the adapters, accepted drafts of
    each request, the labels behind them and their log-probabilities."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device).manual_seed(seed)
    ids = rng.integers(0, sources, samples).astype(np.int32)
    x = rng.integers(0, 256, (samples, n_features)) * (ids + 2)[:, None] // (sources + 1)
    x = torch.from_numpy(x.astype(np.uint8)).to(device)              # sources differ in contrast
    ids = torch.from_numpy(ids).to(device)
    teacher = bl.BitlogicModel.from_numpy(*network(rng, n_features, (4000, 4000), 6),
                                          n_classes, device=device)
    thresholds, layers = network(rng, n_features, (1000, 1000), 6)
    counts, _ = bl.BitlogicModel.from_numpy(thresholds, layers, n_classes,
                                            device=device).forward(x)
    head = np.clip(np.round(100 * np.eye(n_classes) + rng.normal(0, 4, (n_classes, n_classes))),
                   -127, 127).astype(np.int8)
    base, _ = bl.BitlogicModel.from_numpy(thresholds, layers, n_classes, device=device,
                                          head_weights=head).forward(x)
    scores, _ = teacher.forward(x)
    values, classes, log_norm = bl.bitlogic_top_logits(scores, 4, temperature)

    # logits = base / 100 + up (down counts), an adapter a source; up starts at zero
    down = torch.randn(sources, rank, n_classes, device=device, generator=gen)
    down = (down * n_classes ** -0.5).requires_grad_()
    up = torch.zeros(sources, n_classes, rank, device=device, requires_grad=True)
    plan = bl.bitlogic_group_rows(ids, sources)
    optimizer = torch.optim.Adam([down, up], lr=0.005)
    losses = []
    for step in range(steps):
        optimizer.zero_grad()
        dropped = bl.bitlogic_dropout(counts, drop, seed, offset=step)
        logits = bl.bitlogic_adapt(dropped, down, up, ids, 1.0, base, 0.01, plan)
        loss = bl.bitlogic_distill_loss(logits, values, classes, log_norm, temperature,
                                        temperature).mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())

    # labels: a request is drafts + 1 inputs in a row
    requests = samples // (drafts + 1)
    with torch.no_grad():
        logits, _ = bl.bitlogic_adapters(counts, down.detach(), up.detach(), ids, 1.0, base,
                                         0.01, plan)

    def gumbel(*shape):
        return -torch.empty(shape, device=device).exponential_(generator=gen).log()

    drafted, _ = bl.bitlogic_sample(logits, gumbel(samples, n_classes), temperature)

    def by_request(t):
        return t[:requests * (drafts + 1)].view(requests, drafts + 1, *t.shape[1:])

    accepted, token, log_prob = bl.bitlogic_verify(
        by_request(scores), by_request(drafted)[:, :drafts].contiguous(),
        by_request(logits)[:, :drafts],
        torch.rand(requests, drafts, device=device, generator=gen),
        gumbel(requests, n_classes), temperature=temperature)
    return (torch.stack(losses).tolist(), (down.grad, up.grad), accepted, token, log_prob)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--samples", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=60)
    args = ap.parse_args()
    losses, _, accepted, token, log_prob = run(args.samples, args.steps)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} after {args.steps} steps")
    print(f"{token.numel()} requests, {float(accepted.float().mean()):.2f} drafts accepted of 3")
