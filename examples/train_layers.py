"""Two MaxK layers trained full batch on a synthetic graph, their inputs kept in 32, 8 or 4 bits for the backward pass.

    python examples/train_layers.py [--nodes 20000] [--degree 20] [--steps 30]

Every node has one of a few classes; features are its class's direction in noise, edges mostly join nodes of one class.  Prints the loss and what a step
keeps for its backward pass.
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
import paper_2312_08656_amd as maxk  # noqa: E402


def make_graph(nodes: int, degree: int, classes: int, gen: torch.Generator):
    """(graph handle, class of each node): `degree` neighbours a node, four of five of its own class, mean aggregation, self-loops."""
    label = torch.randint(classes, (nodes,), generator=gen, device="cuda")
    order = torch.argsort(label)  # nodes by class
    first = torch.searchsorted(label[order], torch.arange(classes + 1, device="cuda"))
    lo, hi = first[label].unsqueeze(1), first[label + 1].unsqueeze(1)
    u = torch.rand(nodes, degree, generator=gen, device="cuda")
    own = order[(lo + (u * (hi - lo)).long()).clamp(max=nodes - 1)]
    other = torch.randint(nodes, (nodes, degree), generator=gen, device="cuda")
    col = torch.where(torch.rand(nodes, degree, generator=gen, device="cuda") < 0.8, own, other)
    col = torch.cat([torch.arange(nodes, device="cuda").unsqueeze(1), col], dim=1)
    rowptr = torch.arange(0, nodes * (degree + 1) + 1, degree + 1, device="cuda", dtype=torch.int32)
    val = torch.full((nodes * (degree + 1),), 1.0 / (degree + 1), device="cuda")
    return maxk.maxk_graph_create(rowptr, col.reshape(-1).to(torch.int32), val), label


def layer(x, W, b, graph, k, bits):
    if bits == 32:
        return maxk.maxk_aggregate(torch.nn.functional.linear(x, W, b), graph, k)
    return maxk.maxk_layer(x, W, b, graph, k, bits)


def train(bits: int, nodes: int = 20000, degree: int = 20, steps: int = 30, width: int = 256, k: int = 32, classes: int = 16, seed: int = 0):
    """Losses of the steps, and the bytes that a forward pass leaves on the tape."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    graph, label = make_graph(nodes, degree, classes, gen)
    x = 0.4 * torch.randn(classes, 100, generator=gen, device="cuda")[label] + torch.randn(nodes, 100, generator=gen, device="cuda")
    shapes = ((width, 100), (width, width), (classes, width))
    weights = [((torch.rand(s, generator=gen, device="cuda") * 2 - 1) / s[1] ** 0.5).requires_grad_(True) for s in shapes]
    biases = [torch.zeros(s[0], device="cuda", requires_grad=True) for s in shapes]
    optimizer = torch.optim.Adam(weights + biases, lr=3e-3)
    losses, kept = [], 0
    for step in range(steps):
        optimizer.zero_grad(set_to_none=True)
        tape = {}
        with torch.autograd.graph.saved_tensors_hooks(lambda t: (tape.__setitem__(t.data_ptr(), t.numel() * t.element_size()), t)[1], lambda t: t):
            h = layer(x, weights[0], biases[0], graph, k, bits)
            h = layer(h, weights[1], biases[1], graph, k, bits)
        kept = sum(tape.values()) - sum(w.numel() * 4 for w in weights[:2] if w.data_ptr() in tape)
        loss = torch.nn.functional.cross_entropy(torch.nn.functional.linear(h, weights[2], biases[2]), label)
        loss.backward()
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    graph.destroy()
    return losses, kept


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--nodes", type=int, default=20000)
    parser.add_argument("--degree", type=int, default=20)
    parser.add_argument("--steps", type=int, default=30)
    args = parser.parse_args()
    for bits in (32, 8, 4):
        losses, kept = train(bits, args.nodes, args.degree, args.steps)
        print(f"inputs kept in {bits:2d} bits: loss {losses[0]:.4f} -> {losses[-1]:.4f}, two layers keep {kept / 2**20:.1f} MiB for the backward pass", flush=True)


if __name__ == "__main__":
    main()
