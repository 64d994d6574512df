"""Training one temporal layer over nodes of several types, on a small graph.

Nodes are of a few kinds, each with weights of its own: a batch's slots are sampled (Sec. 3.1 of the TGL paper), their
rows looked up and given to their kind's projection, averaged per root, added to the
root's own and normed (Sec. 2.2); the loss asks whether two roots will meet.
Gradients come from torch's autograd, through the operators' own backward passes.

    python examples/train_typed.py [--batches N]
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2203_14883_amd as tgl  # noqa: E402

KINDS, FANOUT = 3, 10


class Layer:
    """Weights of every kind, for a root's own row and for its neighbours'."""

    def __init__(self, dim: int, out: int, device="cuda", seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            return (torch.randn(*shape, device=device, generator=g) / math.sqrt(shape[-1])).requires_grad_()

        self.own, self.near = weight(KINDS, out, dim), weight(KINDS, out, dim)
        self.bias = torch.zeros(KINDS, out, device=device, requires_grad=True)
        self.gamma = torch.ones(out, device=device, requires_grad=True)
        self.beta = torch.zeros(out, device=device, requires_grad=True)
        self.parameters = [self.own, self.near, self.bias, self.gamma, self.beta]

    def __call__(self, rows, kind, roots, slots):
        """Rows of the roots after the layer: ``rows [nodes, dim]``, ``slots [roots, FANOUT]`` with -1 where there is none."""
        flat = slots.reshape(-1)
        # a root and a slot that is padding have no type here and there: their products are zeros
        near = tgl.linear_typed(rows[flat.clamp(min=0).long()], self.near, tgl.group_rows(kind, KINDS, ids=flat))
        count = (slots >= 0).sum(1, keepdim=True).clamp(min=1)
        near = near.view(len(slots), FANOUT, -1).sum(1) / count
        own = tgl.linear_typed(rows[roots.long()], self.own, tgl.group_rows(kind, KINDS, ids=roots), self.bias)
        return tgl.layer_norm(near, self.gamma, self.beta, residual=own)[0]


def loss_of(layer, rows, kind, src, dst, slots):
    """Cross entropy of pairs that met against the same sources with another's destination."""
    z = layer(rows, kind, torch.cat([src, dst]), slots)
    a, b = z[: len(src)], z[len(src):]
    scale = 1 / math.sqrt(z.shape[1])
    met, other = (a * b).sum(1) * scale, (a * b.roll(1, 0)).sum(1) * scale
    return torch.nn.functional.softplus(-met).mean() + torch.nn.functional.softplus(other).mean()


def train(nodes=2000, edges=30_000, batches=20, batch=300, dim=64, out=48, rate=0.1, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    src, dst = (torch.randint(0, nodes, (edges,), device="cuda", generator=g, dtype=torch.int32) for _ in range(2))
    ts = torch.arange(edges, device="cuda", dtype=torch.float32)
    graph = tgl.tcsr_build(src, dst, ts, None, nodes, True)
    kind = torch.randint(0, KINDS, (nodes,), device="cuda", generator=g, dtype=torch.int32)
    rows = torch.randn(nodes, dim, device="cuda", generator=g)
    layer, losses = Layer(dim, out, seed=seed), []
    for i in range(batches):
        at = slice(edges - (batches - i) * batch, edges - (batches - i - 1) * batch)
        times = torch.cat([ts[at], ts[at]])
        slots = tgl.sample(graph, torch.cat([src[at], dst[at]]), times, (FANOUT,), "recent")[0].nbr.view(-1, FANOUT)
        loss = loss_of(layer, rows, kind, src[at], dst[at], slots)
        grads = torch.autograd.grad(loss, layer.parameters)
        with torch.no_grad():
            for p, d in zip(layer.parameters, grads):
                p -= rate * d
        losses.append(float(loss.detach()))
    return layer, dict(rows=rows, kind=kind, src=src[at], dst=dst[at], slots=slots, losses=losses, grads=grads)


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--batches", type=int, default=20)
    result = train(batches=parser.parse_args().batches)[1]
    for n, value in enumerate(result["losses"]):
        print("batch %3d  loss %.4f" % (n, value))
