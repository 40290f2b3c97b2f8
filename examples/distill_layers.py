"""A student of two normed MaxK layers taught by a teacher's likeliest classes, and its last layer served for one node with 4-bit weights.

    python examples/distill_layers.py [--nodes 20000] [--degree 20] [--steps 30] [--temperature 2]

The teacher, two plain layers in 32 bits, learns the classes of a synthetic graph from their log probabilities; what it passes on is its logits of the likeliest few
classes of every node.  The student keeps its layers' inputs in 8 bits, written by the norms in front of them.  Prints both losses and the served node's answer.
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent))
from train_layers import make_graph  # noqa: E402

import paper_2312_08656_amd as maxk  # noqa: E402


def uniform(shape, gen):
    return ((torch.rand(shape, generator=gen, device="cuda") * 2 - 1) / shape[1] ** 0.5).requires_grad_(True)


def train_teacher(graph, x, label, width, k, classes, steps, gen):
    """Losses of the steps, and the logits that it ends with."""
    W = [uniform(s, gen) for s in ((width, x.shape[1]), (width, width), (classes, width))]
    optimizer, losses = torch.optim.Adam(W, lr=3e-3), []
    for _ in range(steps):
        optimizer.zero_grad(set_to_none=True)
        h = maxk.maxk_aggregate(torch.nn.functional.linear(x, W[0]), graph, k)
        h = maxk.maxk_aggregate(torch.nn.functional.linear(h, W[1]), graph, k)
        logits = torch.nn.functional.linear(h, W[2])
        logprob, _ = maxk.maxk_class_logprobs(logits, label)
        loss = -logprob.mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist(), logits.detach()


def student_forward(params, graph, x, k, bits):
    """(logits, hidden features before the last product)."""
    W, b, gamma = params
    h = maxk.maxk_layer(x, W[0], b[0], graph, k, bits)
    out, h = maxk.maxk_norm_layer(h, torch.zeros_like(h), gamma[0], W[1], b[1], graph, k, bits)
    h, _ = maxk.maxk_residual_norm(out, gamma[1], h)
    return torch.nn.functional.linear(h, W[2], b[2]), h


def train(nodes=20000, degree=20, steps=30, width=256, k=32, classes=16, kept=5, temperature=2.0, bits=8, seed=0):
    """(teacher's losses, student's losses, (classes, log probabilities) of node 0 as served)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    graph, label = make_graph(nodes, degree, classes, gen)
    x = 0.4 * torch.randn(classes, 100, generator=gen, device="cuda")[label] + torch.randn(nodes, 100, generator=gen, device="cuda")
    taught, logits = train_teacher(graph, x, label, width, k, classes, steps, gen)
    top_data, top_index = torch.empty(nodes, kept, device="cuda"), torch.empty(nodes, kept, dtype=torch.uint8, device="cuda")
    maxk.maxk_topk_cbsr(logits, kept, top_data, top_index)  # all that the student sees of the teacher

    W = [uniform(s, gen) for s in ((width, x.shape[1]), (width, width), (classes, width))]
    b = [torch.zeros(s.shape[0], device="cuda", requires_grad=True) for s in W]
    gamma = [torch.ones(width, device="cuda", requires_grad=True) for _ in range(2)]
    optimizer, losses = torch.optim.Adam(W + b + gamma, lr=3e-3), []
    for _ in range(steps):
        optimizer.zero_grad(set_to_none=True)
        logits, _ = student_forward((W, b, gamma), graph, x, k, bits)
        loss = maxk.maxk_distill_loss(logits, top_data, top_index, temperature).mean()
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())

    with torch.no_grad():  # node 0: the last product from 4-bit weights, then its likeliest classes
        _, h = student_forward((W, b, gamma), graph, x, k, bits)
        codes, scales = maxk.mx_empty(classes, width, 4)
        maxk.maxk_mx_quantize(W[2].detach(), codes, scales)
        answer, data, index = torch.empty(1, classes, device="cuda"), torch.empty(1, 3, device="cuda"), torch.empty(1, 3, dtype=torch.uint8, device="cuda")
        maxk.maxk_mx_matvec(h[:1].contiguous(), codes, scales, answer, b[2].detach())
        maxk.maxk_logprobs(answer, top_data=data, top_index=index)
    graph.destroy()
    return taught, torch.stack(losses).tolist(), (index[0].tolist(), data[0].tolist())


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--nodes", type=int, default=20000)
    parser.add_argument("--degree", type=int, default=20)
    parser.add_argument("--steps", type=int, default=30)
    parser.add_argument("--temperature", type=float, default=2.0)
    args = parser.parse_args()
    taught, losses, (classes, logprobs) = train(args.nodes, args.degree, args.steps, temperature=args.temperature)
    print(f"teacher: loss {taught[0]:.4f} -> {taught[-1]:.4f}")
    print(f"student: divergence {losses[0]:.4f} -> {losses[-1]:.4f}")
    print("node 0: " + ", ".join(f"class {c} ({p:.3f})" for c, p in zip(classes, logprobs)), flush=True)


if __name__ == "__main__":
    main()
