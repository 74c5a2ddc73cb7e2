"""Fits a linear query encoder to an index whose rows are held in 4 bits.

The teacher is the index's own exact search over the clean queries; the student sees the same queries through a
fixed random distortion and learns the map back:

    q = f W                             (the encoder)
    s = quantised q . quantised rows    (mx_quantize, mx_scores)
    loss, ds = distillation of s towards the teacher's lists      (distill_step)
    dq = ds rows                        (mx_scores_grad)
    dW = f^T dq, a step of Adam

``python examples/fit_queries.py`` prints the loss and the share of the teacher's five best rows that the student's
five best hold, before and after.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_08340_amd as oprag  # noqa: E402

TAU, TEACHER_TAU = 0.05, 0.05


def unit(x):
    return x / x.norm(dim=1, keepdim=True)


def student_scores(features, weight, rows):
    """The encoder's queries, in 6 bits, against the rows."""
    return oprag.mx_scores(oprag.mx_quantize(features @ weight, bits=6), rows)


def recall(scores, teacher_ids, k=5):
    best = scores.topk(k, dim=1).indices
    return (best[:, :, None] == teacher_ids[:, None, :k]).any(dim=2).float().mean().item()


def fit(n=8192, dim=256, batch=256, k=32, steps=60, lr=0.02, seed=1):
    """Returns (mean loss and recall at the start, the same at the end)."""
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    centres = normal(64, dim)
    rows = unit(centres[torch.randint(0, 64, (n,), generator=g, device=dev)] + 0.3 * normal(n, dim))
    index = oprag.Index(dim, n, torch.bfloat16)
    index.upsert(rows)
    few_bits = oprag.mx_quantize(index.rows(), bits=4)  # once: 4.25 bits an element
    distortion = torch.eye(dim, device=dev) + 0.1 * normal(dim, dim)

    def queries():
        clean = unit(rows[torch.randint(0, n, (batch,), generator=g, device=dev)] + 0.3 / dim ** 0.5 * normal(batch, dim))
        t, ids = index.search_dense(clean.to(torch.bfloat16), k)
        return unit(clean @ distortion), ids, t

    weight = torch.eye(dim, device=dev)
    share = torch.full((batch,), 1.0 / batch, device=dev)
    first, second = torch.zeros_like(weight), torch.zeros_like(weight)
    held_out = queries()

    def held_out_quality():
        features, ids, t = held_out
        s = student_scores(features, weight, few_bits)
        loss, _ = oprag.distill_loss(s, ids, t, temperature=TAU, teacher_temperature=TEACHER_TAU)
        return loss.mean().item(), recall(s, ids)

    before = held_out_quality()
    for step in range(1, steps + 1):
        features, ids, t = queries()
        s = student_scores(features, weight, few_bits)
        _, ds = oprag.distill_step(s, ids, t, share, temperature=TAU, teacher_temperature=TEACHER_TAU, out=s)
        dw = features.t() @ oprag.mx_scores_grad(ds, few_bits)
        first.mul_(0.9).add_(dw, alpha=0.1)
        second.mul_(0.99).addcmul_(dw, dw, value=0.01)
        fix1, fix2 = 1 - 0.9 ** step, 1 - 0.99 ** step
        weight -= lr * (first / fix1) / ((second / fix2).sqrt() + 1e-8)
    return before, held_out_quality()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rows", type=int, default=32768)
    ap.add_argument("--dim", type=int, default=512)
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    before, after = fit(a.rows, a.dim, a.batch, steps=a.steps)
    for name, (loss, hits) in (("before", before), ("after", after)):
        print(f"{name}: loss {loss:.4f}, recall at 5 {hits:.3f}")


if __name__ == "__main__":
    main()
