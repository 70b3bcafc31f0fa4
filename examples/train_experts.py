"""A small language model's block trained by synchronous SGD with backup workers, on one GPU.

Each of N + b simulated workers computes the gradient of its own mini-batch with the library's layers (layer norm,
tokens sorted by expert and back) and writes it into its row; the server keeps the first N rows to arrive, moves the
experts' stacked matrices with the orthogonalised update and everything else with momentum.

    python examples/train_experts.py [--steps 30]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1604_00981_b200 import binding as sgdb  # noqa: E402
from paper_1604_00981_b200 import layers  # noqa: E402

TOKENS, WIDTH, HIDDEN, EXPERTS, CHOICES, CLASSES = 256, 64, 96, 4, 2, 32


def shapes():
    """Parameters in the order of a gradient row; the experts' matrices come first."""
    return {"up": (EXPERTS, WIDTH, HIDDEN), "down": (EXPERTS, HIDDEN, WIDTH), "router": (WIDTH, EXPERTS), "embed": (CLASSES, WIDTH),
            "gamma": (WIDTH,), "beta": (WIDTH,), "out": (WIDTH, CLASSES)}


def ranges():
    """First column of each parameter in a row; each begins on a multiple of 64 columns."""
    at, first = 0, {}
    for name, shape in shapes().items():
        first[name] = at
        at += (int(np.prod(shape)) + 63) // 64 * 64
    return first, at


def forward(p, tokens, targets):
    """Mean cross entropy of guessing the next token."""
    x = p["embed"][tokens]
    h = layers.layer_norm(x, p["gamma"], p["beta"])
    top = torch.topk(h @ p["router"], CHOICES, dim=1)
    r = layers.route(top.indices.int().contiguous(), EXPERTS)
    xs = layers.dispatch(h, r)
    edges = r.offsets.tolist()
    ys = [torch.relu(xs[a:b] @ p["up"][e]) @ p["down"][e] for e, (a, b) in enumerate(zip(edges, edges[1:]))]
    y = layers.combine(torch.cat(ys + [xs[edges[-1]:]]), torch.softmax(top.values, 1), r)
    return torch.nn.functional.cross_entropy((x + y) @ p["out"], targets)


def train(steps: int = 30, N: int = 4, b: int = 2, seed: int = 1, dtype=torch.float32):
    dev = torch.device("cuda")
    rng = np.random.Generator(np.random.Philox(seed))
    gen = torch.Generator(device=dev).manual_seed(seed)
    first, P = ranges()
    W = N + b
    theta = torch.zeros(P, device=dev)
    p = {}
    for name, shape in shapes().items():
        p[name] = theta[first[name]:first[name] + int(np.prod(shape))].view(shape)
        p[name].copy_(torch.randn(shape, device=dev, generator=gen) * (1.0 if name == "embed" else shape[-2] ** -0.5 if len(shape) > 1 else 0.0))
    p["gamma"].fill_(1.0)
    momentum = torch.zeros_like(theta)
    grad = torch.zeros(W, P, dtype=dtype, device=dev)
    mask = torch.empty(W, dtype=torch.uint8, device=dev)
    order = torch.empty(N, dtype=torch.int32, device=dev)
    info = torch.empty(2, dtype=torch.int32, device=dev)
    rest = first["router"]  # the experts' matrices end here
    orthogonal = {}
    for name in ("up", "down"):
        E, r, c = shapes()[name]
        opt = sgdb.OrthogonalOpt(lr=0.02, momentum=0.9, scale=max(1.0, r / c) ** 0.5)
        orthogonal[name] = (opt, torch.empty(sgdb.sgdb_step_orthogonal_workspace_bytes(E, r, c), dtype=torch.uint8, device=dev))
    other = sgdb.Opt(kind="momentum", lr=0.1, momentum=0.9)
    successor = torch.randperm(CLASSES, device=dev, generator=gen)  # what there is to learn
    losses = []
    for t in range(steps):
        total = 0.0
        for w in range(W):  # the workers
            tokens = torch.randint(0, CLASSES, (TOKENS,), device=dev, generator=gen)
            leaf = {k: v.detach().requires_grad_() for k, v in p.items()}
            loss = forward(leaf, tokens, successor[tokens])
            loss.backward()
            for name, v in leaf.items():
                grad[w, first[name]:first[name] + v.numel()] = v.grad.reshape(-1)
            total += float(loss.detach())
        losses.append(total / W)
        arrival = torch.from_numpy(rng.lognormal(0.0, 0.3, W).astype(np.float32)).to(dev)
        tags = torch.full((W,), t, dtype=torch.int32, device=dev)
        for name, (opt, workspace) in orthogonal.items():  # the server: one piece of the columns after the other
            E, r, c = shapes()[name]
            piece = slice(first[name], first[name] + E * r * c)
            sgdb.sgdb_step_orthogonal(grad.view(-1)[first[name]:], E, r, c, arrival, tags, t, N, b, theta[piece], momentum[piece], opt, mask,
                                      order, info, workspace, ld=P)
        sgdb.sgdb_step(grad.view(-1)[rest:], P - rest, arrival, tags, t, N, b, theta[rest:], momentum[rest:], None, other, mask, order, info,
                       ld=P)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    losses = train(ap.parse_args().steps)
    print("mean loss of the workers: first %.3f, last %.3f (%d steps)" % (losses[0], losses[-1], len(losses)))
