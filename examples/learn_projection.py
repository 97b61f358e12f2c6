"""Learn a projection for an index: the softmax loss over all vectors, its gradient, orthogonalised updates, then the index itself.

Vectors of 512 components, most of which say nothing about which vector a query belongs to, are to be searched as 64 bytes each.  A
matrix P [512, 64] is learnt from pairs (query, vector): each query's projection is scored against the projections of all vectors,

    loss_i = log sum_j exp(scale q_i P . y_j P) - scale q_i P . y_t P

softmax_loss_grad gives the gradients to both projections (the scores are never kept), two products with the inputs make the
gradient of P of them, orthogonalize makes the step.  The projected vectors go into an Index, other queries are answered from it.

    python examples/learn_projection.py [--vectors 20000] [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1102_3828_amd as pkg  # noqa: E402

D, DIM, USEFUL = 512, 64, 48


def data(n, seed=0, device="cuda"):
    """(vectors [n, D], a function that draws queries for given vectors): what queries share with their vector lies in USEFUL directions."""
    g = torch.Generator(device=device).manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device=device)
    basis = torch.linalg.qr(r(D, D))[0]
    useful, rest = basis[:, :USEFUL], basis[:, USEFUL:]
    kept = r(n, USEFUL)
    noise = lambda m: 2.0 * torch.mm(r(m, D - USEFUL), rest.t())
    vectors = torch.mm(kept, useful.t()) + noise(n)
    queries = lambda ids: torch.mm(kept[ids] + 0.2 * r(len(ids), USEFUL), useful.t()) + noise(len(ids))
    return vectors, queries, g


def learn(vectors, queries, g, steps, rows=1024, rate=0.05, momentum=0.9, dtype=torch.bfloat16):
    """P and the loss of each step."""
    device = vectors.device
    P = torch.linalg.qr(torch.randn((D, DIM), generator=g, device=device))[0]
    y = vectors.to(dtype)
    average = torch.zeros_like(P)
    weight = torch.full((rows,), 1.0 / rows, device=device)
    losses = []
    for step in range(steps):
        targets = torch.randint(0, len(vectors), (rows,), generator=g, device=device)
        q = queries(targets).to(dtype)
        half = P.to(dtype)
        loss, dx, dw = pkg.softmax_loss_grad(torch.mm(q, half), torch.mm(y, half), targets, weight, scale=0.5)
        grad = torch.mm(q.t(), dx) + torch.mm(y.t(), dw)
        average = momentum * average + grad.float()
        P -= rate * (1 - step / steps) * pkg.orthogonalize(average)
        losses.append(loss.mean())
    return P, torch.stack(losses)


def as_bytes(x, low, step):
    return ((x - low) / step).round().clamp(0, 255)


def recall(P, vectors, queries, g, count=1000, lists=64, w=16, kprime=100, k=10):
    """The share of queries with their own vector among the first k answers of an index of the projected vectors."""
    y = torch.mm(vectors, P)
    low, high = y.min(), y.max()
    step = (high - low) / 255
    stored = as_bytes(y, low, step).to(torch.uint8)
    index = pkg.Index(DIM, lists, 8, 8)
    index.train(stored, iters=5)
    index.add(stored, 0)
    index.finalize()
    ids = torch.randint(0, len(vectors), (count,), generator=g, device=vectors.device)
    found, _ = index.search(as_bytes(torch.mm(queries(ids), P), low, step).contiguous(), w, kprime, k)
    index.close()
    return (found == ids[:, None].to(torch.int32)).any(1).float().mean().item()


def main(arguments=None):
    a = argparse.ArgumentParser()
    a.add_argument("--vectors", type=int, default=20000)
    a.add_argument("--steps", type=int, default=60)
    a = a.parse_args(arguments)
    vectors, queries, g = data(a.vectors)
    start = torch.linalg.qr(torch.randn((D, DIM), generator=g, device=vectors.device))[0]
    before = recall(start, vectors, queries, g)
    P, losses = learn(vectors, queries, g, a.steps)
    after = recall(P, vectors, queries, g)
    print(f"loss {losses[0].item():.2f} -> {losses[-1].item():.2f}; queries with their vector among ten answers: {before:.2f} -> {after:.2f}")
    return losses, before, after


if __name__ == "__main__":
    main()
