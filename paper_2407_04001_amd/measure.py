"""Layer costs measured on this GPU, and the search with them.

The default cost of a layer is a FLOP count, as if every layer ran at one rate
(Sec. II, eq. (1)).  On an MI355X a layer norm or a softmax is bound by memory,
a product by its matrix units, and a thin shard of a product loses most of its
rate.  Here each layer is run as the operators of `paper_2407_04001_amd.ops`,
forward and backward, at the shard sizes of each of its configurations, and
the times take the FLOP counts' place; what a cost holds besides (the
partial-sum reduction, and gradient synchronisation where asked for) stays.

    python -m paper_2407_04001_amd.measure --workload w4_transformer --p 8

measures a graph, searches it with both kinds of cost and prints what each
strategy costs under the measured ones.
"""
from __future__ import annotations

import argparse
import json
import time
from typing import NamedTuple

import numpy as np
import torch   # before libpase.so, which then uses the HIP runtime that torch loaded

from . import ops
from .pase import Graph


class Shard(NamedTuple):
    """What one device computes of a layer: `kind` is "product" (rows of each of
    `groups` equal groups, n, k), "norm" (rows, n columns) or "softmax" (rows, n classes)."""
    kind: str
    groups: int
    rows: int
    n: int
    k: int


def layer_kind(vertex: dict) -> dict:
    """The operator of a vertex of a graph dict (`workloads.gen`) and the loop dims
    of each of its sizes.  Raises ValueError for a layer that has none.

    A contraction is a product: of rows and a weight matrix where the layer has
    weights of one word a point; else of two activations, one product for each
    batch element and head (loop dims named b and h).  Without contraction, a
    layer with weights along one loop dim is a layer norm over it, and one with
    work but no weights a softmax over its last loop dim."""
    dims = range(len(vertex["dims"]))
    reduce, weights = set(vertex["reduce"]), set(vertex.get("weight_dims", ()))
    name = vertex["name"]
    if reduce:
        if weights:
            if vertex["weight_per_point"] != 1 or not reduce <= weights:
                raise ValueError(f"{name}: no operator for a contraction with {vertex['weight_per_point']} words a point")
            return {"kind": "product", "groups": [], "rows": [d for d in dims if d not in weights],
                    "n": sorted(weights - reduce), "k": sorted(reduce)}
        names = vertex["dim_names"]
        groups = [d for d in dims if names[d] in ("b", "h") and d not in reduce]
        free = [d for d in dims if d not in reduce and d not in groups]
        if len(free) != 2:
            raise ValueError(f"{name}: no operator for a contraction of two activations over {names}")
        return {"kind": "product", "groups": groups, "rows": free[:1], "n": free[1:], "k": sorted(reduce)}
    if len(weights) == 1:
        return {"kind": "norm", "groups": [], "rows": [d for d in dims if d not in weights], "n": sorted(weights), "k": []}
    if not weights and vertex["flops_per_point"] > 0:
        return {"kind": "softmax", "groups": [], "rows": list(dims)[:-1], "n": [dims[-1]], "k": []}
    raise ValueError(f"{name}: no operator for a layer without contraction, weights or work")


def shard(vertex: dict, splits, kind: dict | None = None) -> Shard:
    """The largest part of a layer under a configuration: each loop dim's size over its split, rounded up."""
    kind = kind or layer_kind(vertex)
    size = [-(-n // s) for n, s in zip(vertex["dims"], splits)]

    def span(ds):
        out = 1
        for d in ds:
            out *= size[d]
        return out

    return Shard(kind["kind"], span(kind["groups"]), span(kind["rows"]), span(kind["n"]), span(kind["k"]))


def training_step(s: Shard, dtype=None):
    """A callable that runs the shard forward and backward once, on inputs made here."""
    dtype = dtype or torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(0)

    def normal(*shape, scale=1.0):
        # drawn for part of a large tensor and repeated: the values do not matter to the time
        n = int(np.prod(shape))
        some = torch.randn(min(n, 1 << 24), generator=gen, device="cuda").mul_(scale).to(dtype)
        return some.repeat(-(-n // some.numel()))[:n].view(shape)

    if s.kind == "product":
        rows = s.groups * s.rows
        x, dy = normal(rows, s.k), normal(rows, s.n)
        w = normal(s.groups, s.n, s.k, scale=s.k ** -0.5)
        offsets = torch.arange(s.groups + 1, dtype=torch.int64, device="cuda") * s.rows

        def step():
            return ops.grouped_matmul_forward(x, w, offsets), ops.grouped_matmul_backward(dy, x, w, offsets)
    elif s.kind == "norm":
        x, residual, dy = normal(s.rows, s.n), normal(s.rows, s.n), normal(s.rows, s.n)
        gain, bias = normal(s.n), normal(s.n)

        def step():
            y, z, mean, rstd = ops.layer_norm_forward(x, gain, bias, residual=residual)
            return y, ops.layer_norm_backward(dy, z, gain, mean, rstd)
    else:
        logits = normal(s.rows, s.n)
        targets = torch.randint(0, s.n, (s.rows,), generator=gen, device="cuda")
        dloss = torch.full((), 1.0 / s.rows, device="cuda")

        def step():
            return ops.softmax_loss_grad(logits, targets, dloss)
    return step


def _sweep():
    """A callable that reads 512 MiB, twice what the caches hold: what was in them before is not after."""
    logits = torch.zeros(1024, 131072, device="cuda")
    targets = torch.zeros(1024, dtype=torch.int32, device="cuda")
    return lambda: ops.softmax_loss_forward(logits, targets)


def step_seconds(step, repeats: int = 3) -> float:
    """Time of one run on the GPU that finds its operands in memory, not in a cache, as
    between the other layers of a training step.  HIP graphs of about a millisecond of runs,
    each after a sweep through the caches, and of the sweeps alone: the least of
    `repeats` replays of the one less that of the other."""
    sweep = _sweep()
    sweep(), step()
    torch.cuda.synchronize()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    begin.record()
    step()
    end.record()
    end.synchronize()
    runs = max(1, min(20, int(1.0 / max(begin.elapsed_time(end), 1e-3))))
    best = []
    for parts in ((sweep,), (sweep, step)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(runs):
                for part in parts:
                    part()
        best.append(float("inf"))
        for _ in range(repeats):
            begin.record()
            graph.replay()
            end.record()
            end.synchronize()
            best[-1] = min(best[-1], begin.elapsed_time(end))
    return max(best[1] - best[0], 1e-3) * 1e-3 / runs


def layer_costs(graph, dtype=None, progress=None):
    """Measured layer costs of a `Graph` whose configurations are enumerated and
    which has been searched once: a list of uint64 arrays, one a vertex, and a dict
    of what was measured.  Times become FLOPs at the rate of the graph's
    largest layer, unsplit, so that they keep their weight against the communication terms."""
    vertices = graph.graph["vertices"]
    kinds = [layer_kind(v) for v in vertices]
    configs = [[graph.config_splits(v, c) for c in range(graph.K[v])] for v in range(graph.nv)]
    shards = [[shard(x, s, k) for s in cs] for x, k, cs in zip(vertices, kinds, configs)]
    flops = [x["flops_per_point"] * int(np.prod([int(n) for n in x["dims"]], dtype=object)) for x in vertices]
    seconds = {}
    todo = sorted({s for per in shards for s in per})
    for i, s in enumerate(todo):
        seconds[s] = step_seconds(training_step(s, dtype))
        if progress and (i + 1) % 100 == 0:
            progress(f"{i + 1} of {len(todo)} shards measured")
    largest = max(range(graph.nv), key=lambda v: flops[v])
    rate = flops[largest] / seconds[shard(vertices[largest], [1] * len(vertices[largest]["dims"]), kinds[largest])]
    costs = []
    for v in range(graph.nv):
        compute = [-(-flops[v] // int(np.prod(c))) for c in configs[v]]
        rest = graph.layer_costs(v).astype(object) - np.array(compute, dtype=object)
        timed = [max(1, round(seconds[s] * rate)) for s in shards[v]]
        costs.append(np.array([int(t) + int(r) for t, r in zip(timed, rest)], np.uint64))
    return costs, {"shards": len(todo), "flops_per_second": rate, "seconds": seconds}


def strategy_cost(graph, layer, edge, strategy) -> int:
    """F of eq. (1) for a strategy under given costs."""
    total = sum(int(layer[v][c]) for v, c in enumerate(strategy))
    for e, d in enumerate(graph.graph["edges"]):
        total += int(edge[e][strategy[d["src"]], strategy[d["dst"]]])
    return total


def search(graph_dict, p: int, dtype=None, progress=None) -> dict:
    """Search a graph with FLOP counts and with measured layer costs."""
    g = Graph(graph_dict)
    g.enumerate_configs(p)
    _, counted = g.find_best_strategy()
    began = time.perf_counter()
    layer, what = layer_costs(g, dtype, progress)
    took = time.perf_counter() - began
    edge = [g.edge_costs(e) for e in range(g.ne)]
    g.override_costs(layer, edge)
    best, measured = g.find_best_strategy()
    return {"graph": graph_dict["name"], "p": p, "shards_measured": what["shards"], "measuring_s": round(took, 2),
            "flops_per_second": what["flops_per_second"], "cost_of_measured_strategy": best,
            "cost_of_counted_strategy": strategy_cost(g, layer, edge, counted),
            "vertices_that_differ": sum(a != b for a, b in zip(counted, measured)),
            "strategy": [g.config_splits(v, c) for v, c in enumerate(measured)], "choice": measured}


def main(argv=None) -> None:
    from workloads.gen import workload
    ap = argparse.ArgumentParser(description="Search a workload with layer costs measured on this GPU.")
    ap.add_argument("--workload", default="w4_transformer", help="w0_fc_chain, w3_lstm_grid or w4_transformer")
    ap.add_argument("--p", type=int, default=8, help="devices (a power of two)")
    a = ap.parse_args(argv)
    out = search(workload(a.workload), a.p, progress=lambda s: print(s, flush=True))
    out.pop("strategy"), out.pop("choice")
    print(json.dumps(out))


if __name__ == "__main__":
    main()
