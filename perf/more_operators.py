"""Performance cases of the operators between a Transformer layer's products:
attention, rotary positions and dropout with the residual's addition, forward
and backward.

One pass of a case is one call a training or decoding step makes for one layer
of a graph (or for one device's shard of it).  Sizes are those of the
Transformer graph of workloads.gen (model width 1024, 16 heads of 64, 64
sequences of 256 tokens), what is left of them on one device where a
configuration splits by three, and generic ones for what that graph has no
lengths for: long ragged sequences with shared heads, and single tokens over
kept keys.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def _at(name, op, sequences, rows, keys, heads, kv_heads, dim, dtype, causal, kind, ragged):
    """kind: "self" (the queries' ranges are the keys'), "cross" (ranges of their own) or "kept"
    (keys at the start of a sequence's own room, more than there are)."""
    c = {"op": op, "sequences": sequences, "rows": rows, "keys": keys, "heads": heads, "kv_heads": kv_heads, "dim": dim,
         "dtype": dtype, "causal": causal, "kind": kind, "ragged": ragged}
    return {"name": name, **c} if name else c


def _ro(name, op, rows, heads, dim, turned, dtype, interleaved, furthest, scaled):
    """turned: elements of a head that are rotated; furthest: one past the largest position."""
    c = {"op": op, "rows": rows, "heads": heads, "dim": dim, "turned": turned, "dtype": dtype, "interleaved": interleaved,
         "furthest": furthest, "scaled": scaled}
    return {"name": name, **c} if name else c


def _dr(name, op, rows, width, dtype, p, residual, pad=0):
    c = {"op": op, "rows": rows, "width": width, "dtype": dtype, "p": p, "residual": residual, "pad": pad}
    return {"name": name, **c} if name else c


def listed():
    return [
        # an encoder layer of the Transformer, whole batch: scores, softmax and context
        _at("attention_forward", "attention", 64, 16384, 16384, 16, 16, 64, "bf16", False, "self", False),
        # a decoder layer's self-attention in the backward pass
        _at("attention_backward", "attention_grad", 64, 16384, 16384, 16, 16, 64, "bf16", True, "self", False),
        # long packed sequences, four heads to one of keys and values
        _at("attention_long_forward", "attention", 4, 16384, 16384, 16, 4, 128, "bf16", True, "self", True),
        _at("attention_long_backward", "attention_grad", 4, 16384, 16384, 16, 4, 128, "bf16", True, "self", True),
        # cross-attention of one device's shard where batch, heads and the head's width are split by three
        _at("attention_cross_third", "attention", 22, 5632, 5511, 6, 6, 22, "fp16", False, "cross", True),
        # decoding: one token of each of 64 sequences
        _at("attention_step", "attention", 64, 64, 131072, 16, 4, 128, "bf16", True, "kept", True),
        # decoding one sequence with much behind it: a single row of work to share out
        _at("attention_step_long", "attention", 1, 1, 131072, 16, 2, 128, "bf16", True, "kept", False),
        # queries and keys of a layer, whole batch
        _ro("rotary_train", "rotary", 16384, 32, 64, 64, "bf16", False, 256, False),
        # one token of each of 64 sequences, far in, half of the head rotated, frequencies scaled: launch latency
        _ro("rotary_step", "rotary", 64, 20, 128, 64, "bf16", True, 1 << 20, True),
        # the gradient in a shard split by three
        _ro("rotary_backward_third", "rotary_grad", 5632, 6, 22, 22, "fp32", False, 256, False),
        # the end of a layer's branch: dropout, then the residual
        _dr("dropout_train", "dropout", 16384, 1024, "bf16", 0.1, True),
        # its gradient on a shard split by three
        _dr("dropout_backward_third", "dropout_grad", 5632, 342, "fp16", 0.1, False),
    ]


def _spread(rng, lo, hi):
    """An integer spread over the logarithm of its range; odd as often as not."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if v > 64 and rng.random() < 0.5:
        v -= v % 64
    return max(lo, min(hi, v))


def draw(rng):
    """One more case: any operator and direction, from one row to a whole batch, one sequence or many, any head
    width up to 128, every type."""
    op = rng.choice(["attention", "attention", "attention_grad", "attention_grad", "rotary", "rotary_grad", "dropout", "dropout_grad"])
    if op == "attention" and rng.random() < 0.4:
        sequences = _spread(rng, 1, 256)
        rows = sequences * rng.choice([1, 1, 1, rng.randint(2, 5)])
        kv_heads, group = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 7, 8])
        dim = rng.choice([64, 128, rng.randint(16, 128)])
        keys = _spread(rng, 1, 131072)
        keys = max(sequences, min(keys, (1 << 26) // (kv_heads * dim)))
        return _at("", op, sequences, rows, keys, kv_heads * group, kv_heads, dim, rng.choice(["bf16", "fp16"]), True, "kept",
                   rng.random() < 0.7)
    if op in ("attention", "attention_grad"):
        sequences = _spread(rng, 1, 64)
        kv_heads, group = rng.choice([1, 2, 4, 6, 16]), rng.choice([1, 1, 2, 4, 7])
        dim = rng.choice([64, 64, 128, 128, rng.randint(16, 128)])
        # (gradients of rows that all see one key are 0 but for what their sums' roundings leave)
        least = 16 if op == "attention_grad" else 1
        rows = max(least * sequences, _spread(rng, 1, 16384))
        # the scores of the longest sequence, each at most, in 2^30 and the products below the largest listed case
        while True:
            longest = min(rows, 3 * rows // sequences + 1)
            if kv_heads * group * longest * longest * sequences <= 1 << 30 and rows * kv_heads * group * dim <= 1 << 25:
                break
            rows = max(least, rows // 2)
            sequences = max(1, min(sequences, rows // least))
        kind = rng.choice(["self", "self", "cross"])
        keys = rows if kind == "self" else max(least * sequences, rows * rng.randint(1, 8) // 8)
        return _at("", op, sequences, rows, keys, kv_heads * group, kv_heads, dim, rng.choice(["bf16", "fp16"]), rng.random() < 0.6,
                   kind, rng.random() < 0.7)
    if op in ("rotary", "rotary_grad"):
        dim = rng.choice([64, 128, rng.randint(2, 128)])
        turned = max(2, rng.choice([dim, dim, dim // 2]) // 2 * 2)
        rows, heads = _spread(rng, 1, 16384), rng.choice([1, 2, 6, 20, 32, 48])
        rows = max(1, min(rows, (1 << 25) // (heads * dim)))
        return _ro("", op, rows, heads, dim, turned, rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.5,
                   rng.choice([256, 8192, 1 << 20, 1 << 26]), rng.random() < 0.5)
    rows, width = _spread(rng, 1, 16384), _spread(rng, 1, 8192)
    rows = max(1, min(rows, (1 << 24) // width))
    return _dr("", op, rows, width, rng.choice(["bf16", "fp16", "fp32"]), rng.choice([0.05, 0.1, 0.3, 0.5]),
               op == "dropout" and rng.random() < 0.7, rng.choice([0, 0, 8, rng.randint(1, 63)]))


def _lengths(total, sequences, ragged, shift=0):
    """`total` dealt to the sequences: evenly, or between 0.3 and 1.7 of the average, in a set order."""
    share = [1.0 + (1.4 * (((i + shift + 1) * 0.6180339887) % 1) - 0.7 if ragged else 0) for i in range(sequences)]
    whole, ends = sum(share), [0]
    for s in share:
        ends.append(ends[-1] + s)
    ends = [round(total * e / whole) for e in ends]
    return [b - a for a, b in zip(ends, ends[1:])]


def _all_lengths(case):
    n, ragged, kind = case["sequences"], case["ragged"], case["kind"]
    q = _lengths(case["rows"], n, ragged and kind != "kept")
    return q, q if kind == "self" else _lengths(case["keys"], n, ragged, 0 if kind == "kept" else 5)


def _room(lengths):
    """Rows that every sequence's kept keys have: the longest, in whole blocks of 64, and one block more."""
    return (max(lengths) + 127) // 64 * 64


# ------------------------------------------------------------------ inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)

    op, dtype = case["op"], TYPES[case["dtype"]]
    if op in ("attention", "attention_grad"):
        rows, n, heads, kv_heads, dim = case["rows"], case["sequences"], case["heads"], case["kv_heads"], case["dim"]
        lq, lk = (torch.tensor(x) for x in _all_lengths(case))
        order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))   # which sequence is the longest: the seed's
        lq, lk = lq[order], lk[order]
        s = {"op": op, "causal": case["causal"], "scale": dim ** -0.5, "most": (int(lq.max()), int(lk.max())), "k_lengths": None}
        s["q_offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), lq.cumsum(0)]).int().cuda()
        if case["kind"] == "kept":
            room = _room(lk.tolist())
            s["k_offsets"] = (torch.arange(n + 1) * room).int().cuda()
            s["k_lengths"] = lk.int().cuda()
            keys = n * room
        else:
            s["k_offsets"] = torch.cat([torch.zeros(1, dtype=torch.int64), lk.cumsum(0)]).int().cuda()
            keys = case["keys"]
        # some queries look for few keys, others at all of them alike
        s["q"] = normal(rows, heads, dim, scale=1.2) * torch.exp(0.3 * normal(rows, heads, 1))
        s["q"] = s["q"].to(dtype)
        # keys and values of a layer come out of one product, side by side
        kv = normal(keys, 2, kv_heads, dim, dtype=dtype)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        if case["kind"] == "kept":   # what no token has been written to yet
            unused = torch.arange(room, device="cuda") >= s["k_lengths"][:, None]
            kv.view(n, room, 2, kv_heads, dim)[unused] = float("nan")
        if op == "attention_grad":
            f = _attention(s)
            s["out"], s["lse"] = f["out"], f["lse"]
            s["dout"] = normal(rows, heads, dim, dtype=dtype, scale=1.0 if case["dtype"] == "fp16" else 0.05)
        return s
    if op in ("rotary", "rotary_grad"):
        rows, heads, dim, turned, furthest = case["rows"], case["heads"], case["dim"], case["turned"], case["furthest"]
        i = torch.arange(turned // 2, dtype=torch.float64, device="cuda")
        f = 10000.0 ** (-2 * i / turned)
        s = {"op": op, "interleaved": case["interleaved"], "magnitude": 1.0}
        if case["scaled"]:   # slow turns stretched 8 times, fast ones kept, those between by parts
            share = ((8192 * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
            f = f / 8 * (1 - share) + f * share
            s["magnitude"] = 0.1 * math.log(8) + 1
        s["frequencies"] = f
        s["positions"] = torch.randint(0, furthest, (rows,), generator=gen, device="cuda")
        s["x"] = normal(rows, heads, dim, dtype=dtype)
        return s
    rows, width, pad = case["rows"], case["width"], case["pad"]
    s = {"op": op, "p": case["p"], "residual": normal(rows, width, dtype=dtype) if case["residual"] else None}
    wide = torch.full((rows, width + pad), float("nan"), dtype=dtype, device="cuda")
    wide[:, :width] = normal(rows, width, dtype=dtype)
    s["x"] = wide[:, :width]
    s["seed"] = torch.randint(-(1 << 63), (1 << 63) - 1, (2,), generator=gen, device="cuda")
    return s


# ------------------------------------------------------------------ the operators
def run(s):
    op = s["op"]
    if own:
        from paper_2407_04001_amd import ops
        if op == "attention":
            out, lse = ops.attention_forward(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], k_lengths=s["k_lengths"],
                                             causal=s["causal"], scale=s["scale"])
            return {"out": out, "lse": lse}
        if op == "attention_grad":
            dq, dk, dv = ops.attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["q_offsets"],
                                                s["k_offsets"], causal=s["causal"], scale=s["scale"])
            return {"dq": dq, "dk": dk, "dv": dv}
        if op == "rotary":
            return ops.rotary_forward(s["x"], s["positions"], s["frequencies"], interleaved=s["interleaved"], magnitude=s["magnitude"])
        if op == "rotary_grad":
            return ops.rotary_backward(s["x"], s["positions"], s["frequencies"], interleaved=s["interleaved"], magnitude=s["magnitude"])
        if op == "dropout":
            return ops.dropout_forward(s["x"], s["p"], s["seed"], residual=s["residual"])
        return ops.dropout_backward(s["x"], s["p"], s["seed"])
    return {"attention": _attention, "attention_grad": _attention_grad, "rotary": _rotary, "rotary_grad": _rotary,
            "dropout": _dropout, "dropout_grad": _dropout}[op](s)


def _places(offsets, lengths, most):
    """Every sequence's rows, padded to the longest: their places [n, most], and which are real."""
    at = torch.arange(most, device=offsets.device)
    real = at < lengths[:, None]
    return torch.where(real, offsets[:-1, None].long() + at, 0), real


def _padded(s, name, places, real, group):
    """q, or k, v: [n, kv_heads, group x most, dim] in 32 bits, 0 where no row is."""
    x = s[name][places].float() * 1.0
    x = torch.where(real[..., None, None], x, 0.0)
    n, most, heads, dim = x.shape
    return x.view(n, most, heads // group, group, dim).permute(0, 2, 3, 1, 4).reshape(n, heads // group, group * most, dim)


def _back(x, places, real, rows, group):
    """The inverse of _padded: [rows, heads, dim]."""
    n, kv_heads, _, dim = x.shape
    most = places.shape[1]
    x = x.view(n, kv_heads, group, most, dim).permute(0, 3, 1, 2, 4).reshape(n, most, kv_heads * group, dim)
    out = torch.zeros(rows, kv_heads * group, dim, device=x.device)
    out[places[real]] = x[real]
    return out


def _scores(s):
    """Scaled scores in 32 bits [n, kv_heads, group x queries, keys], -inf where a key is not seen, and what made them."""
    group = s["q"].shape[1] // s["k"].shape[1]
    lq = s["q_offsets"][1:] - s["q_offsets"][:-1]
    lk = s["k_offsets"][1:] - s["k_offsets"][:-1] if s["k_lengths"] is None else s["k_lengths"]
    (pq, rq), (pk, rk) = _places(s["q_offsets"], lq, s["most"][0]), _places(s["k_offsets"], lk, s["most"][1])
    q, k = _padded(s, "q", pq, rq, group), _padded(s, "k", pk, rk, 1)
    seen = rk[:, None, :].expand(-1, rq.shape[1], -1)
    if s["causal"]:
        i, j = torch.arange(rq.shape[1], device=q.device)[:, None], torch.arange(rk.shape[1], device=q.device)
        seen = seen & (j <= i + (lk - lq)[:, None, None])
    scores = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    scores.view(*scores.shape[:2], group, *seen.shape[1:]).masked_fill_(~seen[:, None, None], float("-inf"))
    return scores, q, k, (pq, rq), (pk, rk), group


def _attention(s):
    scores, q, k, (pq, rq), (pk, rk), group = _scores(s)
    v = _padded(s, "v", pk, rk, 1)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    rows = s["q"].shape[0]
    lse = _back(top + torch.log(total), pq, rq, rows, group)[:, :, 0].t().contiguous()
    return {"out": _back(out, pq, rq, rows, group).to(s["q"].dtype), "lse": lse}


def _attention_grad(s):
    scores, q, k, (pq, rq), (pk, rk), group = _scores(s)
    v = _padded(s, "v", pk, rk, 1)
    dout, out = _padded(s, "dout", pq, rq, group), _padded(s, "out", pq, rq, group)
    lse = _padded({"lse": s["lse"].t()[:, :, None]}, "lse", pq, rq, group)
    p = scores.sub_(torch.where(lse == float("-inf"), 0.0, lse)).exp_()
    dv = torch.matmul(p.transpose(-1, -2), dout)
    ds = torch.matmul(dout, v.transpose(-1, -2)).sub_((dout * out).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(-1, -2), q)
    rows, keys, dtype = s["q"].shape[0], s["k"].shape[0], s["q"].dtype
    return {"dq": _back(dq, pq, rq, rows, group).to(dtype), "dk": _back(dk, pk, rk, keys, 1).to(dtype),
            "dv": _back(dv, pk, rk, keys, 1).to(dtype)}


def _rotary(s):
    x, half = s["x"].float(), s["frequencies"].shape[0]
    angle = s["positions"].double()[:, None] * s["frequencies"]   # far positions need 64 bits
    sign = -1.0 if s["op"] == "rotary_grad" else 1.0
    cos, sin = (angle.cos() * s["magnitude"]).float()[:, None], (angle.sin() * (s["magnitude"] * sign)).float()[:, None]
    turned = x[..., :2 * half]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if s["interleaved"] else (turned[..., :half], turned[..., half:])
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([y, x[..., 2 * half:]], -1).to(s["x"].dtype)


def _numbers(seed, calls):
    """Philox 4x32-10 (Salmon, Moraes, Dror, Shaw 2011): eight 16-bit numbers for each call, of the key
    seed[0] and the counter (call, seed[1]), each 64 bits."""
    low = 0xFFFFFFFF
    key, high = seed[0], seed[1]
    k0, k1 = key & low, (key >> 32) & low
    c0, c1 = calls & low, (calls >> 32) & low
    c2, c3 = (high & low).expand_as(calls), ((high >> 32) & low).expand_as(calls)
    for _ in range(10):   # the generator's ten rounds
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)


def _dropout(s):
    """Element (row, column) takes number column % 8 of call row x ceil(width / 8) + column / 8, and stays
    where it is at least p in units of 2^-16."""
    x = s["x"]
    rows, width = x.shape
    per = -(-width // 8)
    numbers = _numbers(s["seed"], torch.arange(rows * per, device=x.device)).view(rows, per * 8)[:, :width]
    drop = round(s["p"] * 65536)
    y = torch.where(numbers >= drop, x.float() * (65536 / (65536 - drop)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(x.dtype)


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    f8, dev = torch.float64, "cuda"
    if op in ("attention", "attention_grad"):
        heads, dim, group = case["heads"], case["dim"], case["heads"] // case["kv_heads"]
        out = torch.zeros(case["rows"], heads, dim, dtype=f8, device=dev)
        lse = torch.full((heads, case["rows"]), -math.inf, dtype=f8, device=dev)
        dq, dk, dv = torch.zeros_like(out), torch.zeros(s["k"].shape, dtype=f8, device=dev), torch.zeros(s["k"].shape, dtype=f8, device=dev)
        qo, ko = s["q_offsets"].tolist(), s["k_offsets"].tolist()
        lk = s["k_lengths"].tolist() if s["k_lengths"] is not None else [b - a for a, b in zip(ko, ko[1:])]
        for e in range(case["sequences"]):
            rq, rk = slice(qo[e], qo[e + 1]), slice(ko[e], ko[e] + lk[e])
            nq, nk = qo[e + 1] - qo[e], lk[e]
            if not nq or not nk:
                continue
            hidden = None
            if case["causal"]:
                hidden = torch.ones(nq, nk, dtype=torch.bool, device=dev).triu(nk - nq + 1)
            for h in range(heads):
                k, v = s["k"][rk, h // group].to(f8), s["v"][rk, h // group].to(f8)
                q = s["q"][rq, h].to(f8)
                z = torch.mm(q, k.t().contiguous()).mul_(case["dim"] ** -0.5)
                if hidden is not None:
                    z.masked_fill_(hidden, -math.inf)
                if op == "attention":
                    lse[h, rq] = torch.logsumexp(z, 1)
                    out[rq, h] = torch.softmax(z, 1).nan_to_num_(0.0).mm(v)
                    continue
                do, l = s["dout"][rq, h].to(f8), s["lse"][h, rq].to(f8)
                p = torch.exp(z - l.clamp(min=-1e300).unsqueeze(1))
                dv[rk, h // group] += p.t().contiguous() @ do
                # the softmax's derivative along dout . v, with the output that the forward pass gave
                p *= (do @ v.t().contiguous()) - torch.linalg.vecdot(do, s["out"][rq, h].to(f8)).unsqueeze(1)
                dq[rq, h] = p @ k * case["dim"] ** -0.5
                dk[rk, h // group] += p.t().contiguous() @ q * case["dim"] ** -0.5
        return {"out": out, "lse": lse} if op == "attention" else {"dq": dq, "dk": dk, "dv": dv}
    if op in ("rotary", "rotary_grad"):
        # the product with the complex number m e^(i angle), or m e^(-i angle)
        half = case["turned"] // 2
        x = s["x"].to(f8)
        pair = x[..., :2 * half].unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
        pair = pair if case["interleaved"] else pair.transpose(-1, -2)
        turn = torch.outer(s["positions"].to(f8), s["frequencies"])
        turn = torch.polar(torch.full_like(turn, s["magnitude"]), turn if op == "rotary" else -turn).unsqueeze(1)
        y = torch.view_as_real(torch.complex(pair[..., 0], pair[..., 1]) * turn)
        y = y if case["interleaved"] else y.transpose(-1, -2)
        return torch.cat([y.flatten(-2), x[..., 2 * half:]], -1)
    rows, width = case["rows"], case["width"]
    import numpy as np
    words = s["seed"].cpu().numpy().view(np.uint32)
    per = (width + 7) // 8
    c = np.zeros((rows * per, 4), np.uint64)
    c[:, 0], c[:, 2], c[:, 3] = np.arange(rows * per), words[2], words[3]
    key = np.array([words[0], words[1]], np.uint64)
    for step in range(10):
        even = c[:, [2, 0]] * np.array([0xCD9E8D57, 0xD2511F53], np.uint64)
        k = (key + np.uint64(step) * np.array([0x9E3779B9, 0xBB67AE85], np.uint64)) & np.uint64(0xFFFFFFFF)
        c[:, [0, 2]] = (even >> np.uint64(32)) ^ c[:, [1, 3]] ^ k
        c[:, [1, 3]] = even & np.uint64(0xFFFFFFFF)
    numbers = c.astype(np.uint32).view(np.uint16).reshape(rows, per * 8)[:, :width]
    drop = round(case["p"] * 65536)
    keep = torch.from_numpy((numbers >= drop).astype(np.float64)).cuda()
    y = s["x"].to(f8) * keep / (1 - drop / 65536)
    return y if s["residual"] is None else y + s["residual"].to(f8)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op, b = case["op"], BYTES[case["dtype"]]
    if op in ("attention", "attention_grad"):
        seen = 0
        for nq, nk in zip(*_all_lengths(case)):
            if not case["causal"]:
                seen += nq * nk
            else:   # the last query sees all keys, each before it one less
                full = min(nq, nk)
                seen += full * nk - full * (full - 1) // 2
        flops = case["heads"] * case["dim"] * seen
        q, kv, stats = case["rows"] * case["heads"] * case["dim"] * b, case["keys"] * case["kv_heads"] * case["dim"] * b, 4 * case["rows"] * case["heads"]
        if op == "attention":   # two products; q, k, v in, out and one statistic a row out
            return {"bytes": 2 * q + 2 * kv + stats, "flops": 4 * flops}
        # five products; q, out, dout, k, v and the statistic in, three gradients out
        return {"bytes": 4 * q + 4 * kv + stats, "flops": 10 * flops}
    if op in ("rotary", "rotary_grad"):
        return {"bytes": 2 * case["rows"] * case["heads"] * case["dim"] * b + 8 * case["rows"] + 4 * case["turned"],
                "flops": 3 * case["rows"] * case["heads"] * case["turned"]}
    points = case["rows"] * case["width"]
    return {"bytes": points * b * (3 if case["residual"] else 2) + 16, "flops": 2 * points}
