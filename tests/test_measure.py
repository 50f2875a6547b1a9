"""Measured layer costs: the operator and the shard sizes of every kind of layer
(no GPU), and a search with measured costs (GPU)."""
import numpy as np
import pytest

from paper_2407_04001_amd.measure import Shard, layer_kind, shard
from workloads import fc_chain, inception, residual_cnn, workload
from workloads.gen import lstm_grid, transformer


def by_name(g):
    return {v["name"]: v for v in g["vertices"]}


def test_every_layer_of_the_transformer_has_its_operator():
    v = by_name(transformer(enc_layers=1, dec_layers=1))
    whole = {n: shard(x, [1] * len(x["dims"])) for n, x in v.items()}
    rows = 64 * 256
    assert whole["enc0_qkv"] == Shard("product", 1, rows, 16 * 192, 1024)
    assert whole["enc0_score"] == Shard("product", 64 * 16, 256, 256, 64)
    assert whole["enc0_ctx"] == Shard("product", 64 * 16, 256, 64, 256)
    assert whole["enc0_oproj"] == Shard("product", 1, rows, 1024, 1024)
    assert whole["enc0_ln1"] == Shard("norm", 1, rows, 1024, 1)
    assert whole["enc0_ffn1"] == Shard("product", 1, rows, 4096, 1024)
    assert whole["enc0_ffn2"] == Shard("product", 1, rows, 1024, 4096)
    assert whole["dec0_xkv"] == Shard("product", 1, rows, 16 * 128, 1024)
    assert whole["src_emb"] == Shard("product", 1, rows, 1024, 32768)
    assert whole["proj"] == Shard("product", 1, rows, 32768, 1024)
    assert whole["softmax"] == Shard("softmax", 1, rows, 32768, 1)


def test_the_product_of_a_shard_is_the_layers_work():
    """groups x rows x n x k of the unsplit layer are its iteration points, whatever the roles of its loop dims."""
    for g in (transformer(enc_layers=1, dec_layers=1), fc_chain(), lstm_grid(steps=3)):
        for v in g["vertices"]:
            s = shard(v, [1] * len(v["dims"]))
            assert s.groups * s.rows * s.n * s.k == int(np.prod([int(n) for n in v["dims"]], dtype=object)), v["name"]


def test_splits_round_up():
    v = by_name(transformer())
    assert shard(v["enc0_ffn1"], [2, 1, 3, 1]) == Shard("product", 1, 32 * 256, 1366, 1024)
    assert shard(v["enc0_ln1"], [3, 1, 3]) == Shard("norm", 1, 22 * 256, 342, 1)
    assert shard(v["enc0_score"], [4, 1, 2, 1, 5]) == Shard("product", 16 * 8, 256, 256, 13)


@pytest.mark.parametrize("g", [residual_cnn(), inception()], ids=["residual_cnn", "inception"])
def test_convolutions_are_refused(g):
    with pytest.raises(ValueError):
        [layer_kind(v) for v in g["vertices"]]


@pytest.mark.gpu
def test_search_with_measured_costs():
    from paper_2407_04001_amd import Graph, measure
    from oracle.oracle import Oracle
    gd = transformer(p=4, enc_layers=1, dec_layers=1, d_model=64, heads=4, ffn=256, seq=16, batch=4, vocab=512)
    g = Graph(gd)
    g.enumerate_configs(4)
    _, counted = g.find_best_strategy()
    layer, what = measure.layer_costs(g)
    edge = [g.edge_costs(e) for e in range(g.ne)]
    assert [len(c) for c in layer] == g.K and all((c > 0).all() for c in layer)
    assert all(0 < s < 1 for s in what["seconds"].values())
    g.override_costs(layer, edge)
    best, choice = g.find_best_strategy()
    assert best == measure.strategy_cost(g, layer, edge, choice)
    assert best <= measure.strategy_cost(g, layer, edge, counted)
    o = Oracle(gd)
    o.configs(4)
    o.set_costs(layer, edge)
    o.solve()
    assert o.result() == (best, choice)


@pytest.mark.gpu
def test_command(capsys):
    import json

    from paper_2407_04001_amd import measure
    measure.main(["--workload", "w0_fc_chain", "--p", "4"])
    out = json.loads(capsys.readouterr().out.splitlines()[-1])
    assert out["cost_of_measured_strategy"] <= out["cost_of_counted_strategy"]
    assert workload("w0_fc_chain")["name"] == out["graph"]


@pytest.mark.gpu
def test_measured_steps_find_their_operands_in_memory():
    """A layer norm whose operands (100 MB) the caches would hold between two runs takes no less than one that goes
    round eight sets of them, whose outputs alone may still be there (58 us against 70; in the caches 49)."""
    import torch
    from paper_2407_04001_amd import measure
    s = Shard("norm", 1, 16384, 1024, 1)
    steps = [measure.training_step(s) for _ in range(8)]
    for step in steps:
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for step in steps:
            step()
    begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    around = float("inf")
    for _ in range(5):
        begin.record()
        graph.replay()
        end.record()
        end.synchronize()
        around = min(around, begin.elapsed_time(end) * 1e-3 / len(steps))
    assert 0.95 * around <= measure.step_seconds(steps[0]) <= 2 * around
