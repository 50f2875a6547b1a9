"""Performance cases of the layer operators: residual add + layer norm, matrix
products grouped by ragged row ranges, and the softmax loss, forward and
backward.

One pass of a case is one call a training or decoding step makes for one layer
of a graph (or for one device's shard of it).  Sizes are those of the
Transformer and LSTM graphs of workloads.gen: model width 1024, feed-forward
width 4096, 64 sequences of 256 tokens, vocabularies of 32768 and 65536, and
what is left of them on one device where a configuration splits by three.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
IGNORE = -100


def _ln(name, op, rows, width, dtype, param, residual=True, pad=0):
    """pad: columns of the buffer that x is a column slice of, past its own."""
    c = {"op": op, "rows": rows, "width": width, "dtype": dtype, "param": param, "residual": residual, "pad": pad}
    return {"name": name, **c} if name else c


def _gm(name, op, rows, groups, k, n, dtype, grad="", spare=0, pad=0):
    """grad: type of the weights' gradient; spare: rows at the end that belong to no group."""
    c = {"op": op, "rows": rows, "groups": groups, "k": k, "n": n, "dtype": dtype, "grad": grad or dtype,
         "spare": spare, "pad": pad}
    return {"name": name, **c} if name else c


def _sl(name, op, rows, classes, dtype, pad=0):
    c = {"op": op, "rows": rows, "classes": classes, "dtype": dtype, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of each of 64 sequences through a layer norm: launch latency
        _ln("norm_step", "norm", 64, 1024, "bf16", "bf16"),
        # a layer norm vertex of the Transformer, whole batch
        _ln("norm_forward", "norm", 16384, 1024, "bf16", "fp32"),
        # its backward pass, with a second gradient reaching the sum (pre-norm order)
        _ln("norm_backward", "norm_grad", 16384, 1024, "bf16", "fp32"),
        # one device's shard where batch and width are split by three: odd width, single precision
        _ln("norm_backward_third", "norm_grad", 5632, 342, "fp32", "fp32", residual=False),
        # one token of each of 64 sequences through eight experts' first product: the weights' bytes
        _gm("experts_step", "product", 64, 8, 1024, 4096, "bf16"),
        # a feed-forward vertex with eight experts, whole batch
        _gm("experts_forward", "product", 16384, 8, 1024, 4096, "bf16"),
        # its backward pass: both gradients
        _gm("experts_backward", "product_grad", 16384, 8, 1024, 4096, "bf16"),
        # a third of the rows and of the feed-forward width, many small experts, spare rows at the end
        _gm("experts_backward_third", "product_grad", 5632, 32, 1024, 1366, "fp16", grad="fp32", spare=137),
        # the LSTM's projection on its vocabulary, as one group
        _gm("projection_forward", "product", 1280, 1, 2048, 65536, "bf16"),
        # the Transformer's softmax vertex in training, whole batch: loss and gradient
        _sl("loss_train", "loss_grad", 16384, 32768, "bf16"),
        # the LSTM's softmax in evaluation: loss alone
        _sl("loss_eval", "loss", 1280, 65536, "fp32"),
        # a small batch on a third of the vocabulary, padded rows
        _sl("loss_train_third", "loss_grad", 64, 10923, "fp16", pad=5),
    ]


def _spread(rng, lo, hi):
    """An integer spread over the logarithm of its range; odd as often as not."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v > 64 and rng.random() < 0.5:
        v -= v % 64
    return max(lo, min(hi, v))


def draw(rng):
    """One more case: any operator and direction, from one row to a whole
    batch, widths of any remainder, every type, padded buffers."""
    op = rng.choice(["norm", "norm_grad", "product", "product_grad", "loss", "loss_grad"])
    pad = rng.choice([0, 0, 0, 8, rng.randint(1, 63)])
    if op in ("norm", "norm_grad"):
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        rows, width = _spread(rng, 1, 16384), _spread(rng, 16, 8192)
        rows = max(1, min(rows, (1 << 25) // width))
        return _ln("", op, rows, width, dtype, rng.choice([dtype, "fp32"]), rng.random() < 0.7, pad)
    if op in ("product", "product_grad"):
        dtype = rng.choice(["bf16", "fp16"])
        groups = _spread(rng, 1, 64)
        k, n = _spread(rng, 64, 4096), _spread(rng, 64, 8192)
        groups = max(1, min(groups, (1 << 27) // (k * n)))
        rows = _spread(rng, 1, 16384)
        rows = max(1, min(rows, int(6.8e10 / (k * n))))
        spare = rng.choice([0, 0, rng.randint(0, rows // 4)])
        return _gm("", op, rows, groups, k, n, dtype, rng.choice([dtype, "fp32"]), spare, pad)
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    rows, classes = _spread(rng, 1, 16384), _spread(rng, 64, 131072)
    rows = max(1, min(rows, (1 << 28) // classes))
    return _sl("", op, rows, classes, dtype, pad)


# ------------------------------------------------------------------ inputs
def _padded(t, pad):
    """t as a column slice of a wider buffer."""
    if not pad:
        return t
    wide = torch.empty(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=t.device).fill_(float("nan"))
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)

    op, dtype = case["op"], TYPES[case["dtype"]]
    if op in ("norm", "norm_grad"):
        rows, width, param = case["rows"], case["width"], TYPES[case["param"]]
        s = {"op": op, "eps": 1e-5, "gain": normal(width, dtype=param, scale=0.2, shift=1.0)}
        if op == "norm":
            s["bias"] = normal(width, dtype=param, scale=0.2)
            # a residual stream: some columns far larger than the rest, a mean that is not zero
            columns = torch.exp(0.5 * normal(width))
            s["x"] = _padded((normal(rows, width) * columns + 0.3).to(dtype), case["pad"])
            s["residual"] = normal(rows, width, dtype=dtype, scale=0.5) if case["residual"] else None
            return s
        s["z"] = normal(rows, width, dtype=dtype, scale=1.3, shift=0.2)
        z = s["z"].float()
        s["mean"] = z.mean(1)
        s["rstd"] = 1 / torch.sqrt((z - s["mean"][:, None]).square().mean(1) + s["eps"])
        s["dy"] = _padded(normal(rows, width, dtype=dtype, scale=0.05), case["pad"])
        s["dz"] = normal(rows, width, dtype=dtype, scale=0.05) if case["residual"] else None
        return s
    if op in ("product", "product_grad"):
        rows, groups, k, n = case["rows"], case["groups"], case["k"], case["n"]
        # what a router leaves: uneven shares, some experts without a row
        share = torch.exp(0.7 * normal(groups))
        share = share * (torch.rand(groups, generator=gen, device="cuda") > (0.1 if groups > 4 else 0.0)) + 1e-9
        pick = torch.multinomial(share, rows - case["spare"], replacement=True, generator=gen)
        counts = torch.bincount(pick, minlength=groups)
        offsets = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
        offsets[1:] = counts.cumsum(0)
        s = {"op": op, "offsets": offsets, "longest": max(1, int(counts.max())), "grad": TYPES[case["grad"]],
             "w": normal(groups, n, k, dtype=dtype, scale=k ** -0.5)}
        s["x"] = _padded(normal(rows, k, dtype=dtype), case["pad"])
        if op == "product_grad":
            s["dy"] = _padded(normal(rows, n, dtype=dtype, scale=0.1), case["pad"])
        return s
    rows, classes = case["rows"], case["classes"]
    logits = _padded(normal(rows, classes, dtype=dtype, scale=2.5), case["pad"])
    # a constrained row in 50 may not use the upper half of its classes
    cut = torch.rand(rows, generator=gen, device="cuda") < 0.02
    logits[:, classes // 2:].masked_fill_(cut[:, None], float("-inf"))
    targets = torch.randint(0, max(1, classes // 2), (rows,), generator=gen, device="cuda")
    targets[torch.rand(rows, generator=gen, device="cuda") < 0.1] = IGNORE
    s = {"op": op, "logits": logits, "targets": targets}
    if op == "loss_grad":
        # the mean over the rows that count, times the loss scale of half precision
        scale = 1024.0 if case["dtype"] == "fp16" else 1.0
        s["dloss"] = torch.full((rows,), scale / rows, device="cuda")
    return s


# ------------------------------------------------------------------ the operators
def run(s):
    op = s["op"]
    if own:
        from paper_2407_04001_amd import ops
        if op == "norm":
            y, z, mean, rstd = ops.layer_norm_forward(s["x"], s["gain"], s["bias"], residual=s["residual"], eps=s["eps"])
            return {"y": y, "z": z if s["residual"] is not None else None, "mean": mean, "rstd": rstd}
        if op == "norm_grad":
            dx, dgain, dbias = ops.layer_norm_backward(s["dy"], s["z"], s["gain"], s["mean"], s["rstd"], dz=s["dz"])
            return {"dx": dx, "dgain": dgain, "dbias": dbias}
        if op == "product":
            return ops.grouped_matmul_forward(s["x"], s["w"], s["offsets"])
        if op == "product_grad":
            dx, dw = ops.grouped_matmul_backward(s["dy"], s["x"], s["w"], s["offsets"], grad_dtype=s["grad"])
            return {"dx": dx, "dw": dw}
        if op == "loss":
            loss, lse = ops.softmax_loss_forward(s["logits"], s["targets"], ignore_index=IGNORE)
            return {"loss": loss, "lse": lse}
        loss, lse, dlogits = ops.softmax_loss_grad(s["logits"], s["targets"], s["dloss"], ignore_index=IGNORE)
        return {"loss": loss, "lse": lse, "dlogits": dlogits}
    return {"norm": _norm, "norm_grad": _norm_grad, "product": _product, "product_grad": _product_grad,
            "loss": _loss, "loss_grad": _loss}[op](s)


def _norm(s):
    z = s["x"].float()
    if s["residual"] is not None:
        z = z + s["residual"].float()
    mean = z.mean(1)
    centred = z - mean[:, None]
    rstd = 1 / torch.sqrt(centred.square().mean(1) + s["eps"])
    y = centred * rstd[:, None] * s["gain"].float() + s["bias"].float()
    dtype = s["x"].dtype
    return {"y": y.to(dtype), "z": z.to(dtype) if s["residual"] is not None else None, "mean": mean, "rstd": rstd}


def _norm_grad(s):
    dy = s["dy"].float()
    h = (s["z"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dh = dy * s["gain"].float()
    dx = (dh - dh.mean(1, keepdim=True) - h * (dh * h).mean(1, keepdim=True)) * s["rstd"][:, None]
    if s["dz"] is not None:
        dx = dx + s["dz"].float()
    param = s["gain"].dtype
    return {"dx": dx.to(s["dy"].dtype), "dgain": (dy * h).sum(0).to(param), "dbias": dy.sum(0).to(param)}


def _ranges(s, rows):
    """Every group's rows, padded to the longest group: their places [E, L] and
    which of them are real; and every row's place in that layout, and whether
    it has one."""
    offsets = s["offsets"].long()
    places = offsets[:-1, None] + torch.arange(s["longest"], device=offsets.device)
    real = places < offsets[1:, None]
    row = torch.arange(rows, device=offsets.device)
    group = (torch.searchsorted(offsets, row, right=True) - 1).clamp(0, len(offsets) - 2)
    inside = row < offsets[-1]
    back = torch.where(inside, group * s["longest"] + row - offsets[group], 0)
    return places.clamp(max=rows - 1), real, back, inside


def _product(s):
    places, real, back, inside = _ranges(s, s["x"].shape[0])
    x = s["x"].float()[places] * real[..., None]
    y = torch.bmm(x, s["w"].float().transpose(1, 2)).flatten(0, 1)[back]
    return torch.where(inside[:, None], y, 0.0).to(s["x"].dtype)


def _product_grad(s):
    places, real, back, inside = _ranges(s, s["x"].shape[0])
    x = s["x"].float()[places] * real[..., None]
    dy = s["dy"].float()[places] * real[..., None]
    dx = torch.bmm(dy, s["w"].float()).flatten(0, 1)[back]
    dw = torch.bmm(dy.transpose(1, 2), x)
    return {"dx": torch.where(inside[:, None], dx, 0.0).to(s["x"].dtype), "dw": dw.to(s["grad"])}


def _loss(s):
    logits = s["logits"].float()
    counts = s["targets"] != IGNORE
    target = s["targets"].clamp(min=0)
    top = logits.amax(1, keepdim=True)
    lse = top[:, 0] + torch.log(torch.exp(logits - top).sum(1))
    loss = lse - logits.gather(1, target[:, None])[:, 0]
    out = {"loss": torch.where(counts, loss, 0.0), "lse": torch.where(counts, lse, 0.0)}
    if s["op"] == "loss_grad":
        dloss = torch.where(counts, s["dloss"], 0.0)[:, None]
        d = torch.exp(logits - lse[:, None]) * dloss
        d.scatter_add_(1, target[:, None], -dloss)
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f8 = torch.float64
    if op == "norm":
        z = s["x"].to(f8) + (s["residual"].to(f8) if s["residual"] is not None else 0)
        var, mean = torch.var_mean(z, dim=1, correction=0)
        rstd = (var + s["eps"]) ** -0.5
        y = torch.addcmul(s["bias"].to(f8), (z - mean.unsqueeze(1)) * rstd.unsqueeze(1), s["gain"].to(f8))
        return {"y": y, "z": z if s["residual"] is not None else None, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        # the derivative of sum(y dy) through the given statistics' formulas: the projections of dy g on 1 and on h
        d = case["width"]
        r = s["rstd"].to(f8).unsqueeze(1)
        h = (s["z"].to(f8) - s["mean"].to(f8).unsqueeze(1)) * r
        g = s["dy"].to(f8) * s["gain"].to(f8)
        dx = r / d * (d * g - g.sum(1, keepdim=True) - h * torch.linalg.vecdot(g, h, dim=1).unsqueeze(1))
        if s["dz"] is not None:
            dx += s["dz"].to(f8)
        return {"dx": dx, "dgain": torch.linalg.vecdot(s["dy"].to(f8), h, dim=0), "dbias": s["dy"].to(f8).sum(0)}
    if op in ("product", "product_grad"):
        ends = s["offsets"].tolist()
        spans = [(e, slice(a, b)) for e, (a, b) in enumerate(zip(ends, ends[1:])) if b > a]
        if op == "product":
            y = torch.zeros(case["rows"], case["n"], dtype=f8, device="cuda")
            for e, span in spans:
                y[span] = s["x"][span].to(f8) @ s["w"][e].to(f8).t().contiguous()
            return y
        dx = torch.zeros(case["rows"], case["k"], dtype=f8, device="cuda")
        dw = torch.zeros(case["groups"], case["n"], case["k"], dtype=f8, device="cuda")
        for e, span in spans:
            dy = s["dy"][span].to(f8)
            dx[span] = dy @ s["w"][e].to(f8)
            dw[e] = dy.t().contiguous() @ s["x"][span].to(f8)
        return {"dx": dx, "dw": dw}
    rows, classes = case["rows"], case["classes"]
    out = {"loss": torch.zeros(rows, dtype=f8, device="cuda"), "lse": torch.zeros(rows, dtype=f8, device="cuda")}
    if op == "loss_grad":
        out["dlogits"] = torch.zeros(rows, classes, dtype=f8, device="cuda")
    at = torch.nonzero(s["targets"] != IGNORE)[:, 0]
    for part in at.split(1024):
        l, t = s["logits"][part].to(f8), s["targets"][part]
        one = torch.arange(len(part), device="cuda")
        lse = torch.logsumexp(l, 1)
        out["lse"][part] = lse
        out["loss"][part] = lse - l[one, t]
        if op == "loss_grad":
            p = (l - lse.unsqueeze(1)).exp()
            p[one, t] -= 1
            out["dlogits"][part] = p * s["dloss"][part].to(f8).unsqueeze(1)
    return out


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, b = case["op"], BYTES[case["dtype"]]
    if op in ("norm", "norm_grad"):
        points, params = case["rows"] * case["width"], case["width"] * BYTES[case["param"]]
        if op == "norm":   # x (and the residual) in, y (and the sum) out, two statistics a row
            return {"bytes": points * b * (4 if case["residual"] else 2) + 8 * case["rows"] + 2 * params, "flops": 8 * points}
        # dy, z (and dz) in, dx out
        return {"bytes": points * b * (4 if case["residual"] else 3) + 8 * case["rows"] + 3 * params, "flops": 14 * points}
    if op in ("product", "product_grad"):
        rows, used, groups, k, n = case["rows"], case["rows"] - case["spare"], case["groups"], case["k"], case["n"]
        live = min(groups, used)   # groups that have rows, at most
        if op == "product":
            return {"bytes": b * (used * k + live * n * k + rows * n) + 4 * (groups + 1), "flops": 2 * used * k * n}
        return {"bytes": b * (used * (k + n) + live * n * k + rows * k) + BYTES[case["grad"]] * groups * n * k
                + 4 * (groups + 1), "flops": 4 * used * k * n}
    points = case["rows"] * case["classes"]
    rest = case["rows"] * (8 + 8)   # targets in; loss and log-sum-exp out
    if op == "loss":
        return {"bytes": points * b + rest, "flops": 4 * points}
    return {"bytes": 2 * points * b + rest + 4 * case["rows"], "flops": 7 * points}
