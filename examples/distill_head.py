"""Fit the quantized head of a small LUT network to a wider network's scores.

A wide network is the teacher: its GroupSum scores are cut to each sample's top few
(bitlogic_top_logits).  The student is a smaller network whose counts go through a
c x c head; the head's float weights are fitted against the teacher's lists
(bitlogic_distill_loss) by gradient descent, snapped to int8 and deployed in the
student (the quantized head of BitlogicModel).  Labels are then drawn from the
deployed network's logits (bitlogic_sample), as one does for pseudo-labels.

    python examples/distill_head.py [--samples N] [--steps K]

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


def run(samples=8192, steps=60, n_features=784, n_classes=10, temperature=8.0, seed=0,
        device="cuda"):
    """Returns the losses of the fit, the deployed network's loss and the drawn labels."""
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.integers(0, 256, (samples, n_features), dtype=np.uint8)).to(device)
    teacher = bl.BitlogicModel.from_numpy(*network(rng, n_features, (4000, 4000), 6),
                                          n_classes, device=device)
    thresholds, layers = network(rng, n_features, (1000, 1000), 6)
    student = bl.BitlogicModel.from_numpy(thresholds, layers, n_classes, device=device)

    # what the teacher hands on: its top scores, their classes, and the mass they leave out
    scores, _ = teacher.forward(x)
    values, classes, log_norm = bl.bitlogic_top_logits(scores, 4, temperature)

    # the head: logits = counts W^T, and W starts at the identity (the popcount head)
    counts = student.forward(x)[0].float()
    weights = torch.eye(n_classes, device=device, requires_grad=True)
    optimizer = torch.optim.Adam([weights], lr=0.005)
    losses = []
    for _ in range(steps):
        optimizer.zero_grad()
        loss = bl.bitlogic_distill_loss(counts @ weights.t(), values, classes, log_norm,
                                        temperature, temperature).mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())

    # deploy: int8 weights, and a temperature that undoes their scale
    scale = 127 / weights.detach().abs().max()
    quantized = torch.round(weights.detach() * scale).to(torch.int8).cpu().numpy()
    deployed = bl.BitlogicModel.from_numpy(thresholds, layers, n_classes, device=device,
                                           head_weights=quantized)
    logits, _ = deployed.forward(x)
    at = temperature * float(scale)
    deployed_loss, _ = bl.bitlogic_distill(logits, values, classes, log_norm, at, temperature,
                                           want_grad=False)

    # labels drawn from the deployed network
    gen = torch.Generator(device).manual_seed(seed)
    noise = -torch.empty(logits.shape, device=device).exponential_(generator=gen).log()
    labels, log_prob = bl.bitlogic_sample(logits, noise, at, top_k=5, top_p=0.95)
    return torch.stack(losses).tolist(), float(deployed_loss.mean()), labels, log_prob


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--samples", type=int, default=8192)
    ap.add_argument("--steps", type=int, default=60)
    args = ap.parse_args()
    losses, deployed, labels, log_prob = run(args.samples, args.steps)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} after {args.steps} steps, "
          f"{deployed:.4f} with the int8 head")
    print(f"{labels.numel()} labels drawn, mean log-probability {float(log_prob.mean()):.3f}")
