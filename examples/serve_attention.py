"""Serving one temporal attention layer in 8 bits, on a Wikipedia-shaped graph.

A node's state is a row (its memory, Sec. 2.1 of the TGL paper); the layer
attends from a root to its neighbours with keys and values made from theirs
(Sec. 2.2).  Both ways of keeping keys and values are shown:

* by node: one token per node, overwritten when the node's row changes; a root
  attends over the neighbours that the sampler picked, whose ids are the
  pages (keys of the neighbour's state alone: the edge and the time between
  root and slot are one per slot, for which a node's page has no room);
* by history: a node's events one after another in pages of 16, their keys made
  with the time since the last one; a root attends over the newest of its own past.

    python examples/serve_attention.py [--batches N] [--edges N]
"""
import argparse
import math
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2203_14883_amd as tgl  # noqa: E402
from paper_2203_14883_amd import workloads  # noqa: E402

DIM, TIME, HEADS, HEAD = 172, 100, 2, 50        # the paper's widths for Wikipedia
PAGE, FANOUT, WINDOW = 16, 10, 256


class Layer:
    """Weights in 8 bits, rounded once, and the caches they fill."""

    def __init__(self, num_nodes: int, max_events: int, max_roots: int, device="cuda", seed: int = 0):
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(out, inner):
            return tgl.quant_rows(torch.randn(out, inner, device=device, generator=g) / math.sqrt(inner))

        width = HEADS * HEAD
        self.norm = torch.ones(DIM, device=device)
        self.qkv = weight(3 * width, DIM)
        self.out = weight(DIM, width)
        self.event_kv = weight(2 * width, DIM + TIME)
        self.omega = torch.logspace(0, -9, TIME, device=device)
        self.phi = torch.zeros(TIME, device=device)
        self.nodes = tgl.HistoryCache.empty(num_nodes, HEADS, HEAD, 1, device)
        # every node's history gets its own pages, so many that none runs out
        self.pages_per_node = (max_events + PAGE - 1) // PAGE
        self.history = tgl.HistoryCache.empty(num_nodes * self.pages_per_node, HEADS, HEAD, PAGE, device)
        self.table = torch.arange(num_nodes * self.pages_per_node, dtype=torch.int32, device=device).view(num_nodes, -1)
        self.length = torch.zeros(num_nodes, dtype=torch.int64, device=device)
        self.sampler = tgl.Sampler(max_roots, (FANOUT,), 1, device)

    def project(self, rows, change=None):
        """Queries, keys and values of rows: [n, HEADS, HEAD] each, and the rows with their change added."""
        q8, scale, rows_now = tgl.norm_quant(rows, self.norm, residual=change)
        y = tgl.linear_i8(q8, scale, *self.qkv, out_dtype=rows.dtype).view(len(rows), 3, HEADS, HEAD)
        return y[:, 0], y[:, 1], y[:, 2], rows if change is None else rows_now

    def update_nodes(self, ids, rows):
        """Keys and values of nodes whose rows have changed (each id once)."""
        _, k, v, _ = self.project(rows)
        tgl.cache_write(self.nodes, k, v, ids.view(-1, 1))

    def attend(self, graph, roots, times, rows):
        """The layer's output for roots at times: attention over sampled neighbours and over the root's own past."""
        self.sampler.run(graph, roots, times, mode="recent")
        slots = self.sampler.nbr[0][:roots.numel() * FANOUT].view(-1, FANOUT)       # -1: no neighbour
        q, _, _, _ = self.project(rows)
        near = tgl.cache_attend(self.nodes, q, slots)
        end = self.length[roots.long()]
        past = tgl.cache_attend(self.history, q, self.table[roots.long()], begin=(end - WINDOW).clamp(min=0), end=end)
        both = (near + past).reshape(len(rows), HEADS * HEAD)
        return tgl.linear_i8(*tgl.quant_rows(both), *self.out, out_dtype=rows.dtype)

    def append_events(self, ids, rows, dt):
        """One new event for each of these nodes (each id once), dt after its last."""
        x = torch.cat([rows, tgl.time_encode(dt, self.omega, self.phi, out_dtype=rows.dtype)], 1)
        kv = tgl.linear_i8(*tgl.quant_rows(x), *self.event_kv, out_dtype=rows.dtype).view(len(rows), 2, HEADS, HEAD)
        at = ids.long()
        tgl.cache_write(self.history, kv[:, 0], kv[:, 1], self.table[at], start=self.length[at])
        self.length[at] += 1


def serve(edges: int = 157_474, batches: int = 20, batch: int = 600, seed: int = 0, device="cuda", dtype=torch.bfloat16):
    """Serves the graph's last batches; the layer, and the outputs of the last one with its roots and times."""
    w = workloads.make_c2(num_edges=edges, seed=seed)
    up = lambda a: torch.from_numpy(a).to(device)  # noqa: E731
    src, dst, ts = up(w.src), up(w.dst), up(w.ts)
    graph = tgl.tcsr_build(src, dst, ts, None, w.num_nodes, True)
    layer = Layer(w.num_nodes, max_events=batches, max_roots=2 * batch, device=device, seed=seed)
    with torch.no_grad():
        g = torch.Generator(device=device).manual_seed(seed + 1)
        memory = torch.randn(w.num_nodes, DIM, device=device, generator=g).to(dtype)
        layer.update_nodes(torch.arange(w.num_nodes, dtype=torch.int32, device=device), memory)
        seen = torch.zeros(w.num_nodes, device=device)
        torch.cuda.synchronize()
        began, out = time.perf_counter(), None
        for i in range(batches):
            e0 = max(0, edges - (batches - i) * batch)
            e1 = min(edges, e0 + batch)
            roots = torch.cat([src[e0:e1], dst[e0:e1]])
            times = torch.cat([ts[e0:e1], ts[e0:e1]])
            out = layer.attend(graph, roots, times, memory[roots.long()])
            # the batch's nodes change: their rows, their keys and values, their histories
            ids, where = torch.unique(roots, return_inverse=True)
            change = torch.zeros(len(ids), DIM, device=device, dtype=torch.float32)
            change.index_add_(0, where, out.float() * 0.1)
            now = torch.zeros(len(ids), device=device).scatter_reduce_(0, where, times, "amax", include_self=False)
            at = ids.long()
            _, _, _, rows = layer.project(memory[at], change.to(dtype))
            memory[at] = rows
            layer.update_nodes(ids, rows)
            layer.append_events(ids, rows, (now - seen[at]).clamp(min=0))
            seen[at] = now
        torch.cuda.synchronize()
        spent = time.perf_counter() - began
    return layer, dict(out=out, roots=roots, times=times, memory=memory, graph=graph, seconds=spent, nodes=w.num_nodes)


def main():
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--batches", type=int, default=20)
    p.add_argument("--edges", type=int, default=157_474)
    a = p.parse_args()
    layer, last = serve(edges=a.edges, batches=a.batches)
    bytes_held = layer.nodes.data.numel() + layer.history.data.numel()
    print("%d batches of %d roots in %.2f ms each; %d nodes and their histories in %.1f MB of 8-bit keys and values"
          % (a.batches, last["roots"].numel(), 1e3 * last["seconds"] / a.batches, last["nodes"], bytes_held / 1e6))


if __name__ == "__main__":
    main()
