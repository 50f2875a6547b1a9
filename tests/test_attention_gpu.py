"""Attention, rotary positions and dropout on the GPU against their definitions in 64 bits.

Tolerances are bounds.  With u the unit roundoff of a matrix's type and e = 2^-24 that of
fp32: a sum of n fp32 terms is off by at most 2 n e times the sum of their magnitudes
(the matrix unit may truncate), a score so by 2 (dim + 8) e scale sum |q k|, and the weight
2^(c s - c m) of it by that, by 4 e (|s| + |m|) for the exponent's own roundings and by 2^-21
for the power, all relative.  Weights (and ds) are rounded to the type once more, by u of each
(fp16: at least half the spacing of its subnormals), and the result by u."""
import math

import pytest
import torch

from test_operators_gpu import BF, E, HF, INF, SF, TINY, U, close, gen, ops, rand, refused  # noqa: F401

pytestmark = pytest.mark.gpu


def bounds(lengths, before=0):
    """Offsets of ranges that begin `before` rows in."""
    out = [before]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def offsets(lengths, before=0, dtype=torch.int32):
    return torch.tensor(bounds(lengths, before), dtype=dtype, device="cuda")


def sequences(q_offsets, k_offsets, k_lengths):
    qo, ko = q_offsets.tolist(), k_offsets.tolist()
    kl = k_lengths.tolist() if k_lengths is not None else [b - a for a, b in zip(ko, ko[1:])]
    return [(slice(a, b), slice(c, c + n)) for a, b, c, n in zip(qo, qo[1:], ko, kl)]


def scores64(q, k, causal, scale):
    """Scores in 64 bits, -inf where a key is not seen, and sum |q k| scale."""
    s = q.double() @ k.double().t() * scale
    size = q.double().abs() @ k.double().abs().t() * scale
    if causal:
        n, m = s.shape
        s = s.masked_fill(torch.ones(n, m, dtype=torch.bool, device=s.device).triu(m - n + 1), -INF)
    return s, size


def weight_error(s, size, top, dim):
    """Of 2^(c (s - top)), relative."""
    seen = s.isfinite()
    return torch.where(seen, 2 * (dim + 8) * E * size + 4 * E * (s.abs() + top.abs()), 0.0) + 2.0 ** -21


def check_forward(got, q, k, v, qo, ko, kl=None, causal=False, scale=None):
    out, lse = got
    rows, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    group = heads // k.shape[1]
    u = U[q.dtype]
    for h in range(heads):
        want, wlse = torch.zeros(rows, dim, dtype=torch.double, device="cuda"), torch.full((rows,), -INF, dtype=torch.double, device="cuda")
        tol, ltol = torch.zeros_like(want), torch.zeros_like(wlse)
        for a, b in sequences(qo, ko, kl):
            n = b.stop - b.start
            if a.stop == a.start or n == 0:
                continue
            s, size = scores64(q[a, h], k[b, h // group], causal, scale)
            l = torch.logsumexp(s, 1)
            empty = l == -INF
            w = torch.where(empty[:, None], 0.0, torch.exp(s - torch.where(empty, 0.0, l)[:, None]))
            vv = v[b, h // group].double()
            err = weight_error(s, size, l[:, None].nan_to_num(0, 0, 0), dim).amax(1, keepdim=True)
            want[a], wlse[a] = w @ vv, l
            av = w @ vv.abs()
            tol[a] = av * (u + 2 * err + 4 * (n + 8) * E) + (TINY[q.dtype] * vv.abs().sum(0) if q.dtype is HF else 0.0) * ~empty[:, None]
            ltol[a] = torch.where(empty, 0.0, err[:, 0] + (n + 8) * E + 8 * E * l.abs())
        close(out[:, h], want, tol, f"out of head {h}")
        close(lse[h], wlse, ltol, f"lse of head {h}")


def check_backward(got, dout, q, k, v, out, lse, qo, ko, kl=None, causal=False, scale=None):
    rows, heads, dim = q.shape
    scale = dim ** -0.5 if scale is None else scale
    group = heads // k.shape[1]
    u, tiny = U[q.dtype], TINY[q.dtype]
    f8 = dict(dtype=torch.double, device="cuda")
    wk, wv = torch.zeros(k.shape, **f8), torch.zeros(k.shape, **f8)
    tk, tv = torch.zeros(k.shape, **f8), torch.zeros(k.shape, **f8)
    for h in range(heads):
        wq, tq = torch.zeros(rows, dim, **f8), torch.zeros(rows, dim, **f8)
        for a, b in sequences(qo, ko, kl):
            n, m = a.stop - a.start, b.stop - b.start
            if n == 0 or m == 0:
                continue
            qq, kk, vv, gg = q[a, h].double(), k[b, h // group].double(), v[b, h // group].double(), dout[a, h].double()
            s, size = scores64(q[a, h], k[b, h // group], causal, scale)
            l = lse[h, a].double()[:, None]
            p = torch.where(l == -INF, 0.0, torch.exp(s - l.nan_to_num(0, 0, 0)))
            perr = p * weight_error(s, size, l.nan_to_num(0, 0, 0), dim)
            dp, delta = gg @ vv.t(), (gg * out[a, h].double()).sum(1, keepdim=True)
            derr = 2 * (dim + 8) * E * (gg.abs() @ vv.abs().t() + (gg.abs() * out[a, h].double().abs()).sum(1, keepdim=True)) + 4 * E * (dp - delta).abs()
            ds = p * (dp - delta)
            seen = s.isfinite()
            serr = ds.abs() * (u + 2 * E) + perr * (dp - delta).abs() + (p + perr) * derr + tiny * seen
            wq[a] = scale * (ds @ kk)
            tq[a] = scale * ((serr + 2 * (m + 8) * E * ds.abs()) @ kk.abs()) + 2 * E * wq[a].abs()
            wk[b, h // group] += scale * (ds.t() @ qq)
            tk[b, h // group] += scale * ((serr + 2 * (n * group + 8) * E * ds.abs()).t() @ qq.abs()) + 2 * E * (scale * (ds.t() @ qq)).abs()
            wv[b, h // group] += p.t() @ gg
            tv[b, h // group] += (perr + p * (u + 2 * (n * group + 8) * E) + tiny * seen).t() @ gg.abs()
        close(got[0][:, h], wq, tq, f"dq of head {h}")
    close(got[1], wk, tk, "dk")
    close(got[2], wv, tv, "dv")


def laid_out(t, layout):
    """t [rows, heads, dim] with other strides, NaN between."""
    rows, heads, dim = t.shape
    if layout == "heads first":
        b = torch.full((heads, rows + 1, dim), float("nan"), dtype=t.dtype, device="cuda")
        b = b.transpose(0, 1)[:rows]
    elif layout == "odd":
        b = torch.full((rows, heads, dim + 3), float("nan"), dtype=t.dtype, device="cuda")[:, :, 1:dim + 1]
    elif layout == "fused":
        b = torch.full((rows, 3, heads + 2, dim), float("nan"), dtype=t.dtype, device="cuda")[:, 1, 1:heads + 1]
    else:
        return t
    b.copy_(t)
    return b


def make(seed, q_lens, k_lens, heads, kv_heads, dim, dtype, room=0, before=0, after=0, layout="", wide=torch.int32):
    """room: key rows a sequence has past its length (k_lengths are then given), all NaN."""
    g = gen(seed)
    rows = before + sum(q_lens) + after
    q = laid_out(rand(g, rows, heads, dim, dtype=dtype, scale=1.3), layout)
    qo = offsets(q_lens, before, wide)
    if room:
        ko = offsets([n + room for n in k_lens], before, wide)
        kl = torch.tensor(k_lens, dtype=wide, device="cuda")
    else:
        ko, kl = offsets(k_lens, before, wide), None
    keys = int(ko[-1]) + after
    k, v = rand(g, keys, kv_heads, dim, dtype=dtype), rand(g, keys, kv_heads, dim, dtype=dtype)
    owned = torch.zeros(keys, dtype=torch.bool, device="cuda")
    for _, b in sequences(qo, ko, kl):
        owned[b] = True
    k[~owned], v[~owned] = float("nan"), float("nan")   # what no sequence may read
    return q, laid_out(k, layout), laid_out(v, layout), qo, ko, kl


CASES = [
    # q lengths, k lengths, heads, kv heads, dim, causal, rest
    ([1], [1], 1, 1, 1, False, {}),
    ([1], [1], 1, 1, 64, True, {}),
    ([3, 0, 2], [5, 4, 0], 2, 1, 8, False, {}),
    ([64], [64], 2, 2, 64, True, {}),
    ([128], [128], 1, 1, 128, True, {}),
    ([127, 129], [127, 129], 3, 3, 64, True, {"before": 5, "after": 7}),
    ([31, 33, 65], [63, 64, 65], 4, 2, 64, False, {}),
    ([200, 1, 0, 77], [130, 300, 9, 0], 4, 2, 128, True, {"before": 2, "after": 1}),
    ([100], [40], 2, 2, 64, True, {}),                       # the first 60 queries see nothing
    ([300], [129], 6, 2, 128, True, {}),
    ([257], [511], 7, 1, 128, True, {"layout": "fused"}),
    ([150, 150], [150, 150], 6, 6, 22, False, {}),
    ([70, 60], [80, 90], 4, 4, 13, True, {}),
    ([70, 60], [80, 90], 2, 1, 40, True, {"layout": "fused"}),
    ([90, 130], [90, 130], 4, 2, 96, True, {"layout": "heads first"}),
    ([65, 64], [65, 64], 2, 2, 64, True, {"layout": "odd"}),
    ([140], [201], 2, 1, 127, False, {"layout": "odd"}),
    ([66, 3], [200, 31], 4, 4, 32, True, {"room": 13}),
    ([65, 64], [65, 64], 2, 2, 22, True, {"layout": "fused"}),   # heads that end inside 16 bytes, NaN behind them
    ([140, 70], [201, 70], 4, 2, 118, True, {"layout": "fused", "room": 9}),
    ([600], [600], 4, 1, 58, True, {"layout": "fused"}),         # few tiles, many steps
    ([600], [600], 4, 1, 128, True, {"layout": "heads first"}),
    ([1500, 0, 1900], [1500, 7, 1900], 4, 1, 64, True, {"before": 3, "after": 2}),   # several sequences of many tiles
    ([520] * 100 + [900], [1100] * 101, 1, 1, 32, True, {"room": 1}),
    ([550, 60], [600, 70], 4, 1, 126, False, {"layout": "fused", "room": 3}),
    ([5, 4, 0, 1], [64, 1, 3, 0], 4, 2, 64, True, {"room": 64, "wide": torch.int64}),
    ([17] * 70, [19] * 70, 2, 2, 16, True, {}),               # more sequences than a wave has lanes
    ([2] * 300 + [0] * 50 + [1] * 4100, [3] * 4450, 1, 1, 32, True, {}),
]
IDS = [f"{len(c[0])}x{c[0][0]}-{c[1][0]}_h{c[2]}-{c[3]}_d{c[4]}{'_causal' if c[5] else ''}{''.join('_' + str(k) for k in c[6])}" for c in CASES]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_attention_forward(ops, case, dtype):  # noqa: F811
    *sizes, causal, rest = case
    q, k, v, qo, ko, kl = make(len(case[0]) + sum(case[0]), *sizes, dtype, **rest)
    check_forward(ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=causal), q, k, v, qo, ko, kl, causal)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_attention_backward(ops, case, dtype):  # noqa: F811
    *sizes, causal, rest = case
    q, k, v, qo, ko, kl = make(1 + sum(case[1]), *sizes, dtype, **rest)
    dout = rand(gen(5), *q.shape, dtype=dtype, scale=0.5)
    out, lse = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=causal)
    got = ops.attention_backward(dout, q, k, v, out, lse, qo, ko, k_lengths=kl, causal=causal)
    check_backward(got, dout, q, k, v, out, lse, qo, ko, kl, causal)


STEPS = [
    # single tokens and a few over kept keys: the keys are shared out
    ([1], [3000], 8, 2, 128, {}),
    ([1], [5], 2, 2, 64, {"room": 4000}),
    ([1, 1, 1], [700, 0, 2049], 16, 4, 128, {"room": 100}),
    ([3, 0, 1, 5], [1000, 50, 3, 1], 4, 4, 64, {"room": 900, "before": 3, "after": 2}),
    ([2, 1], [999, 1500], 14, 2, 80, {"layout": "odd"}),
    ([40], [4096], 3, 1, 32, {}),
    ([1] * 64, [300 + 7 * i for i in range(64)], 4, 1, 64, {"room": 5}),
    ([1] * 20, [128] * 20, 2, 1, 22, {"room": 200}),
    ([1, 2], [3000, 900], 4, 2, 106, {"layout": "fused", "room": 5}),
    ([1, 3], [2000, 900], 4, 2, 30, {"layout": "odd"}),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("case", STEPS, ids=[f"{len(c[0])}x{c[0][0]}-{c[1][0]}_h{c[2]}-{c[3]}_d{c[4]}" for c in STEPS])
def test_attention_of_few_queries(ops, case, dtype):  # noqa: F811
    *sizes, rest = case
    q, k, v, qo, ko, kl = make(sum(case[1]), *sizes, dtype, **rest)
    for causal in (True, False):
        check_forward(ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=causal), q, k, v, qo, ko, kl, causal)


# ------------------------------------------------------------------ rotary positions
def rotary64(x, positions, frequencies, interleaved, magnitude, inverse=False):
    half = frequencies.shape[0]
    t = positions.double()[:, None] * frequencies
    cos, sin = magnitude * t.cos()[:, None], magnitude * (-t.sin() if inverse else t.sin())[:, None]
    y = x.double().clone()
    a, b = (x[..., 0:2 * half:2].double(), x[..., 1:2 * half:2].double()) if interleaved else (x[..., :half].double(), x[..., half:2 * half].double())
    a, b = a * cos - b * sin, a * sin + b * cos
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = a, b
    else:
        y[..., :half], y[..., half:2 * half] = a, b
    return y


def rotary_tolerance(x, half, interleaved, positions, frequencies, magnitude):
    """Sine and cosine in fp32: 4 e of their size and 2^-27 turns of the rest's rounding, the angle's fp64 product 2^-51 of
    itself; the magnitude, two products and a sum: 4 e of each term."""
    pair = torch.zeros_like(x, dtype=torch.double)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    size = (a.double().abs() + b.double().abs()) * magnitude
    angle = 2.0 ** -51 * positions.double().abs()[:, None, None] * frequencies
    tol = size * (8 * E + 2 * math.pi * 2.0 ** -27 + angle)
    if interleaved:
        pair[..., 0:2 * half:2], pair[..., 1:2 * half:2] = tol, tol
    else:
        pair[..., :half], pair[..., half:2 * half] = tol, tol
    return pair


ROTARY = [(1, 1, 2, 2), (5, 3, 22, 22), (7, 1, 13, 6), (64, 20, 128, 64), (33, 2, 128, 128), (1000, 4, 64, 64), (3, 2, 100, 96),
          (700, 1, 8, 2), (2, 5, 300, 258), (600, 3, 31, 30)]


@pytest.mark.parametrize("dtype", [BF, HF, SF])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,turned", ROTARY)
def test_rotary(ops, rows, heads, dim, turned, interleaved, dtype):  # noqa: F811
    g = gen(rows + dim)
    frequencies = ops.rotary_frequencies(turned, factor=4.0, trained=4096)
    for layout, wide, far in (("", torch.int64, 1 << 40), ("heads first", torch.int32, 1 << 20), ("odd", torch.int32, 300), ("fused", torch.int64, 1 << 20)):
        x = laid_out(rand(g, rows, heads, dim, dtype=dtype), layout)
        positions = torch.randint(-far // 4, far, (rows,), generator=g, device="cuda").to(wide)
        for inverse, magnitude in ((False, 1.0), (True, 1.25)):
            call = ops.rotary_backward if inverse else ops.rotary_forward
            want = rotary64(x, positions, frequencies, interleaved, magnitude, inverse)
            tol = rotary_tolerance(x, turned // 2, interleaved, positions, frequencies, magnitude)
            got = call(x, positions, frequencies, interleaved=interleaved, magnitude=magnitude)
            close(got, want, tol, layout)
            assert torch.equal(got[..., turned:], x[..., turned:])
            # the same in place, and into another layout
            y = laid_out(x.clone(), "odd")
            assert call(y, positions, frequencies, interleaved=interleaved, magnitude=magnitude, out=y) is y
            assert torch.equal(y, got)


def test_rotary_frequencies(ops):  # noqa: F811
    f = ops.rotary_frequencies(8, base=100.0)
    assert torch.allclose(f, torch.tensor([1, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.double, device="cuda"), rtol=1e-15)
    assert torch.equal(ops.rotary_frequencies(8, base=100.0, factor=4.0), f / 4)
    # 100 positions trained: 15.9, 5.03, 1.59 and 0.503 turns; kept above 8, divided below 2
    g = ops.rotary_frequencies(8, base=100.0, factor=4.0, trained=100, slow=2.0, fast=8.0)
    share = (100 * 100 ** -0.25 / (2 * math.pi) - 2) / 6
    want = torch.stack([f[0], f[1] * share + f[1] / 4 * (1 - share), f[2] / 4, f[3] / 4])
    assert torch.allclose(g, want, rtol=1e-14)
    for bad in (lambda: ops.rotary_frequencies(7), lambda: ops.rotary_frequencies(0), lambda: ops.rotary_frequencies(8, factor=0.0),
                lambda: ops.rotary_frequencies(8, trained=10, slow=3.0, fast=2.0)):
        assert refused(ops, bad)


# ------------------------------------------------------------------ dropout
def keep_of(rows, width, p, seed):
    """Which elements stay, by the definition on the CPU."""
    from test_attention import philox
    drop = round(p * 65536)
    per = -(-width // 8)
    key, high = (int(s) & (1 << 64) - 1 for s in seed.tolist())
    out = torch.zeros(rows, per * 8, dtype=torch.bool)
    for call in range(rows * per):
        words = philox([call & 0xffffffff, call >> 32, high & 0xffffffff, high >> 32], [key & 0xffffffff, key >> 32])
        numbers = [n for w in words for n in (w & 0xffff, w >> 16)]
        out[call // per, call % per * 8:call % per * 8 + 8] = torch.tensor([n >= drop for n in numbers])
    return out[:, :width].cuda(), drop


@pytest.mark.parametrize("dtype", [BF, HF, SF])
@pytest.mark.parametrize("rows,width,pad", [(1, 1, 0), (3, 7, 0), (5, 8, 3), (2, 65, 8), (40, 342, 0), (9, 1024, 1), (300, 16, 0)])
def test_dropout(ops, rows, width, pad, dtype):  # noqa: F811
    from test_operators_gpu import wide
    g = gen(rows * width)
    x, r = wide(rand(g, rows, width, dtype=dtype), pad), wide(rand(g, rows, width, dtype=dtype), 8 - pad % 8)
    seed = torch.randint(-(1 << 62), 1 << 62, (2,), generator=g, device="cuda")
    for p in (0.0, 0.1, 0.5, 1e-6, 1.0):
        keep, drop = keep_of(rows, width, p, seed)
        scale = 65536 / (65536 - drop) if drop < 65536 else 0.0
        want = torch.where(keep, x.double() * scale, 0.0)
        close(ops.dropout_backward(x, p, seed), want, 2 * E * want.abs(), "dx")
        close(ops.dropout_forward(x, p, seed, residual=r), want + r.double(), 3 * E * (want.abs() + r.double().abs()), "y")
    x[:] = torch.where(keep_of(rows, width, 0.5, seed)[0], x, float("nan"))   # dropped values have no influence
    assert ops.dropout_forward(x, 0.5, seed).isfinite().all()


def test_dropout_keeps_its_share(ops):  # noqa: F811
    """Of n elements n (1 - p) stay, give or take 6 standard deviations, and other seeds give other masks."""
    ones = torch.ones(2048, 4096, device="cuda")
    n = ones.numel()
    kept = []
    for p, seed in ((0.1, [1, 2]), (0.1, [1, 3]), (0.1, [2, 2]), (0.5, [-1, 0])):
        y = ops.dropout_forward(ones, p, torch.tensor(seed, device="cuda"))
        p = round(p * 65536) / 65536
        assert abs(int((y != 0).sum()) - n * (1 - p)) < 6 * math.sqrt(n * p * (1 - p))
        assert (y[y != 0] == 1 / (1 - p)).all() or torch.allclose(y[y != 0], torch.full((), 1 / (1 - p), device="cuda"), rtol=2 * E)
        kept.append(y != 0)
    for a, b in ((0, 1), (0, 2), (1, 2)):   # both kept: 0.81 of all where they are independent
        assert abs(int((kept[a] & kept[b]).sum()) / n - 0.81) < 0.001


# ------------------------------------------------------------------ more of attention
def test_gradients_by_differences(ops):  # noqa: F811
    """dq, dk, dv, and the rotation's and dropout's gradients, against central differences of the 64-bit definition along
    random directions (of the sum of out * dout, in fp16: forward roundings stay out of the differences)."""
    g = gen(31)
    q, k, v, qo, ko, _ = make(31, [9, 5], [12, 5], 4, 2, 24, HF)
    dout = rand(g, *q.shape, dtype=HF)

    def value(q, k, v):
        total = torch.zeros((), dtype=torch.double, device="cuda")
        for a, b in sequences(qo, ko, None):
            for h in range(4):
                s, _ = scores64(q[a, h], k[b, h // 2], True, 24 ** -0.5)
                total += (torch.softmax(s, 1) @ v[b, h // 2].double() * dout[a, h].double()).sum()
        return total

    out, lse = ops.attention_forward(q, k, v, qo, ko, causal=True)
    grads = ops.attention_backward(dout, q, k, v, out, lse, qo, ko, causal=True)
    base = [t.double() for t in (q, k, v)]
    for i in range(3):
        for _ in range(3):
            d = torch.randn(base[i].shape, generator=g, device="cuda", dtype=torch.double)
            e = 1e-5
            up, down = ([t + (s * e * d if j == i else 0) for j, t in enumerate(base)] for s in (1, -1))
            slope = (value(*up) - value(*down)) / (2 * e)
            # the difference's own error is e^2 times a third derivative of order 1; each gradient element is off by about its
            # tolerance of 6 roundings (out, p and ds among them) of the largest terms
            size = (grads[i].double().abs() * d.abs()).sum()
            assert (slope - (grads[i].double() * d).sum()).abs() <= 6 * U[HF] * size + 1e-6 * size


def decoder_layer(O, x, w, gain, offsets, rows_off, positions, frequencies, seeds, p):
    """A decoder layer with causal self-attention: products, rotation, attention, dropout, norm, feed-forward."""
    rows, width = x.shape
    heads, kv, dim = 4, 2, 32
    qkv = O.grouped_matmul(x, w[0], rows_off).view(rows, heads + 2 * kv, dim)
    qk = O.rotary(qkv[:, :heads + kv], positions, frequencies)
    ctx = O.attention(qk[:, :heads], qk[:, heads:], qkv[:, heads + kv:], offsets, offsets, causal=True)
    y = O.grouped_matmul(ctx.reshape(rows, heads * dim), w[1], rows_off)
    z = O.dropout(y, p, seeds[0], residual=x)
    n = O.layer_norm(z, gain[0])
    f = O.grouped_matmul(torch.relu(O.grouped_matmul(n, w[2], rows_off)), w[3], rows_off)
    return O.layer_norm(O.dropout(f, p, seeds[1], residual=n), gain[1])


class Plain:
    """The same in 64-bit torch operations."""

    def __init__(self, rows, width, seeds, p):
        self.keep = [keep_of(rows, width, p, s) for s in seeds]
        self.turn = 0

    @staticmethod
    def grouped_matmul(x, w, offsets):
        return x @ w[0].t()

    @staticmethod
    def rotary(x, positions, frequencies):
        t = positions.double()[:, None] * frequencies
        half = frequencies.shape[0]
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * t.cos()[:, None] - b * t.sin()[:, None], a * t.sin()[:, None] + b * t.cos()[:, None]], -1)

    @staticmethod
    def attention(q, k, v, qo, ko, causal):
        out = []
        for a, b in sequences(qo, ko, None):
            for h in range(q.shape[1]):
                s = q[a, h] @ k[b, h // 2].t() * q.shape[2] ** -0.5
                s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -INF)
                out.append(torch.softmax(s, 1) @ v[b, h // 2])
        n = q.shape[1]
        return torch.cat([torch.stack(out[i:i + n], 1) for i in range(0, len(out), n)])

    def dropout(self, x, p, seed, residual):
        keep, drop = self.keep[self.turn]
        self.turn += 1
        return residual + torch.where(keep, x * (65536 / (65536 - drop)), 0.0)

    @staticmethod
    def layer_norm(x, gain):
        return torch.nn.functional.layer_norm(x, x.shape[1:], gain)


def layer_inputs(dtype, rows=80, width=128):
    g = gen(41)
    lens = [33, 1, 46]
    x = rand(g, rows, width, dtype=dtype)
    w = [rand(g, 1, n, k, dtype=dtype, scale=k ** -0.5) for n, k in ((256, width), (width, 128), (192, width), (width, 192))]
    gain = [rand(g, width, dtype=dtype, scale=0.1, shift=1.0) for _ in range(2)]
    positions = torch.cat([torch.arange(n, device="cuda") for n in lens])
    seeds = torch.randint(-(1 << 60), 1 << 60, (2, 2), generator=g, device="cuda")
    dy = rand(g, rows, width, dtype=dtype)
    return x, w, gain, offsets(lens), offsets([rows]), positions, seeds, dy


def test_a_decoder_layer_and_its_gradients(ops):  # noqa: F811
    """All operators together, as a layer of a model calls them, through torch.autograd, against 64 bits."""
    x, w, gain, off, rows_off, positions, seeds, dy = layer_inputs(HF)
    frequencies = ops.rotary_frequencies(32)
    p = 0.25
    mine = [t.clone().requires_grad_() for t in (x, *w, *gain)]
    y = decoder_layer(ops, mine[0], mine[1:5], mine[5:], off, rows_off, positions, frequencies, seeds, p)
    y.backward(dy)
    plain = [t.double().requires_grad_() for t in (x, *w, *gain)]
    want = decoder_layer(Plain(*x.shape, seeds, p), plain[0], plain[1:5], plain[5:], off, rows_off, positions, frequencies, seeds, p)
    want.backward(dy.double())
    # each of about a dozen operators on the way rounds its results to half precision, by 2^-11 of their size at most; norms
    # over the whole tensor, where these roundings are independent, stay below their sum
    assert (y.double() - want).norm() <= 12 * U[HF] * want.norm()
    for m, t in zip(mine, plain):
        assert (m.grad.double() - t.grad).norm() <= 24 * U[HF] * t.grad.norm()


def passes(ops, x, w, off, few_off, rows_off, positions, frequencies, seeds, dy, p=0.25):  # noqa: F811
    """The passes of the first half of that layer, forward and backward, as a captured training step makes them."""
    rows = x.shape[0]
    qkv = ops.grouped_matmul_forward(x, w[0], rows_off).view(rows, 8, 32)
    qk = ops.rotary_forward(qkv[:, :6], positions, frequencies)
    ctx, lse = ops.attention_forward(qk[:, :4], qk[:, 4:], qkv[:, 6:], off, off, causal=True)
    y = ops.grouped_matmul_forward(ctx.view(rows, 128), w[1], rows_off)
    z = ops.dropout_forward(y, p, seeds[0], residual=x)
    d = ops.dropout_backward(dy, p, seeds[0])
    dctx, dw = ops.grouped_matmul_backward(d, ctx.view(rows, 128), w[1], rows_off)
    dq, dk, dv = ops.attention_backward(dctx.view(rows, 4, 32), qk[:, :4], qk[:, 4:], qkv[:, 6:], ctx, lse, off, off, causal=True)
    dqk = ops.rotary_backward(torch.cat([dq, dk], 1), positions, frequencies)
    few, few_lse = ops.attention_forward(qk[:2, :4], qk[:, 4:], qkv[:, 6:], few_off, off, causal=False)
    return [qkv, qk, ctx, lse, z, dctx, dw, dq, dk, dv, dqk, few, few_lse]


def test_another_stream_and_graph_replays_of_these(ops):  # noqa: F811
    """The same results on a side stream, and from every replay of a captured graph, with other seeds too."""
    x, w, _, off, rows_off, positions, seeds, dy = layer_inputs(BF)
    frequencies, few_off = ops.rotary_frequencies(32), offsets([2, 0, 0])

    def run():
        return passes(ops, x, w, off, few_off, rows_off, positions, frequencies, seeds, dy)

    want = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run()
        with torch.cuda.graph(other, stream=side):   # a second graph, with workspaces of its own
            out2 = run()
    torch.cuda.synchronize()
    kept = x.clone()
    for turn in range(4):
        x.copy_(kept * (1 + turn))
        seeds.add_(turn)
        eager = [t.clone() for t in run()]
        for t in out + out2:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), turn
        assert all(torch.equal(a, b) for a, b in zip(out2, eager)), turn


def test_shares_in_a_captured_graph(ops):  # noqa: F811
    """One token over many kept keys: the shares' workspace is the graph's own."""
    q, k, v, qo, ko, kl = make(51, [1, 1], [3000, 1], 8, 2, 64, BF, room=1096)
    want = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out, lse = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=True)
    for n in (3000, 1, 0, 4096, 77):   # lengths change between replays
        kl[0] = n
        k.view(-1)[:] = k.nan_to_num(0.25).view(-1)
        v.view(-1)[:] = v.nan_to_num(0.25).view(-1)
        want = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=True)
        out.fill_(float("nan")), lse.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), n
        check_forward((out, lse), q, k, v, qo, ko, kl, True)


def test_runs_agree(ops):  # noqa: F811
    """No sum depends on scheduling: the same bits from every run."""
    q, k, v, qo, ko, _ = make(61, [700, 333, 1], [700, 333, 1], 8, 2, 64, BF)
    dout = rand(gen(62), *q.shape, dtype=BF)
    first = None
    for _ in range(5):
        out, lse = ops.attention_forward(q, k, v, qo, ko, causal=True)
        got = [out, lse, *ops.attention_backward(dout, q, k, v, out, lse, qo, ko, causal=True)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


@pytest.mark.parametrize("dim,layout", [(64, ""), (128, ""), (24, "odd"), (128, "odd"), (22, ""), (22, "fused"), (118, "fused"), (60, "fused")])
def test_values_that_are_not_finite_stay_where_they_may(ops, dim, layout):  # noqa: F811
    """What lies past a sequence's length or in other sequences and heads has no influence, whatever it is."""
    g = gen(71)
    q, k, v, qo, ko, kl = make(71, [70, 3, 50], [40, 90, 64], 4, 2, dim, BF, room=30, layout=layout)
    clean = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl)
    dout = rand(g, *q.shape, dtype=BF)
    clean += ops.attention_backward(dout, q, k, v, *clean, qo, ko, k_lengths=kl)
    for bad in (INF, -INF, float("nan"), torch.finfo(BF).min):
        q2, k2, v2, d2 = (t.clone() for t in (q, k, v, dout))
        owned = torch.zeros(k.shape[0], dtype=torch.bool, device="cuda")
        for _, b in sequences(qo, ko, kl):
            owned[b] = True
        k2[~owned], v2[~owned] = bad, bad
        # the second sequence, and the second pair of heads everywhere
        a, b = sequences(qo, ko, kl)[1]
        q2[a], k2[b], v2[b], d2[a] = bad, bad, bad, bad
        q2[:, 2:], k2[:, 1:], v2[:, 1:], d2[:, 2:] = bad, bad, bad, bad
        got = ops.attention_forward(q2, k2, v2, qo, ko, k_lengths=kl)
        got += ops.attention_backward(d2, q2, k2, v2, *got, qo, ko, k_lengths=kl)
        rows = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
        rows[a] = False
        keys = torch.ones(k.shape[0], dtype=torch.bool, device="cuda")
        keys[b] = False
        assert torch.equal(got[0][rows, :2], clean[0][rows, :2]) and torch.equal(got[1][:2, rows], clean[1][:2, rows])
        assert torch.equal(got[2][rows, :2], clean[2][rows, :2])
        for i in (3, 4):
            assert torch.equal(got[i][keys, :1], clean[i][keys, :1])
            assert (got[i][keys & ~owned] == 0).all()


def test_scores_of_any_size(ops):  # noqa: F811
    """Large scores overflow nothing, ties are shared evenly, and one far above the rest takes all."""
    for scale in (1e-6, 1.0, 100.0):
        q, k, v, qo, ko, _ = make(81, [130], [200], 2, 2, 64, HF)
        check_forward(ops.attention_forward(q, k, v, qo, ko, scale=scale), q, k, v, qo, ko, scale=scale)
        q, k, v, qo, ko, _ = make(81, [3], [2000], 2, 2, 64, HF)
        check_forward(ops.attention_forward(q, k, v, qo, ko, scale=scale), q, k, v, qo, ko, scale=scale)
    # rising scores move the reference again and again
    q, k, v, qo, ko, _ = make(82, [100], [1000], 1, 1, 32, BF)
    q[:] = 1.0
    k[:] = torch.linspace(-8, 8, 1000, device="cuda").to(BF)[:, None, None]
    got = ops.attention_forward(q, k, v, qo, ko, scale=2.0)
    check_forward(got, q, k, v, qo, ko, scale=2.0)
    k[:] = 0.0
    got = ops.attention_forward(q, k, v, qo, ko)   # all alike: the mean
    assert torch.allclose(got[0].double(), v.double().mean(0).expand(100, 1, 32), atol=2.0 ** -7, rtol=2.0 ** -8)
    assert torch.allclose(got[1], torch.full((), math.log(1000), device="cuda"), rtol=4 * E)


def test_attention_past_32_bits(ops):  # noqa: F811
    """Rows whose elements are more than 2^31 apart, in the few-query and the many-query kernel and the gradient."""
    heads, dim, keys = 16, 128, (1 << 31) // (16 * 128) + 3000
    g = gen(91)
    kv = torch.zeros(keys, heads, dim, dtype=BF, device="cuda")
    last = slice(keys - 700, keys)
    kv[last] = rand(g, 700, heads, dim, dtype=BF)
    small = kv[last].contiguous()
    so = offsets([0, 700, 0])
    for n in (1, 300, 2200):   # shares, shares of longer tiles, whole tiles of 128 queries
        q = rand(g, n, heads, dim, dtype=BF)
        qo = offsets([0, n, 0])
        ko = torch.tensor([0, keys - 700, keys, keys], dtype=torch.int64, device="cuda").int()
        got = ops.attention_forward(q, kv, kv, qo, ko, causal=True)
        check_forward(got, q, small, small, qo, so, None, True)
        if n > 1:
            dq, dk, dv = ops.attention_backward(q, q, kv, kv, *got, qo, ko, causal=True)
            check_backward((dq, dk[last], dv[last]), q, q, small, small, *got, qo, so, None, True)
            assert (dk[:keys - 700] == 0).all() and (dv[:keys - 700] == 0).all()
    del kv
    # the rotation and dropout at the end of a buffer of that size
    x = torch.zeros((1 << 31) // 2048 + 5, 16, 128, dtype=BF, device="cuda")
    x[-3:] = rand(g, 3, 16, 128, dtype=BF)
    positions = torch.arange(x.shape[0], device="cuda")
    f = ops.rotary_frequencies(128)
    y = ops.rotary_forward(x, positions, f)
    assert torch.equal(y[-3:], ops.rotary_forward(x[-3:].contiguous(), positions[-3:], f)) and (y[:-3] == 0).all()
    seed = torch.tensor([5, 6], device="cuda")
    flat = x.view(-1, 2048)
    z = ops.dropout_forward(flat, 0.5, seed)
    keep = z[-3:] != 0
    assert torch.equal(z[-3:], torch.where(keep, flat[-3:] * 2, 0)) and 2000 < int(keep.sum()) < 4100
    call = (flat.shape[0] - 1) * 256   # the last row's first call: beyond 2^27 calls and 2^31 elements
    from test_attention import philox
    words = philox([call, 0, 6, 0], [5, 0])
    assert [bool(b) for b in z[-1, :8] != 0] == [n >= 32768 for w in words for n in (w & 0xffff, w >> 16)]


def test_offsets_out_of_rule(ops):  # noqa: F811
    """Offsets and lengths outside their ranges are taken as the nearest within; where they decrease, rows of others are left
    alone at least: nothing outside the outputs is written and nothing hangs."""
    q, k, v, qo, ko, _ = make(101, [40, 60], [70, 50], 2, 1, 64, BF)
    want = ops.attention_forward(q, k, v, qo, ko, k_lengths=torch.tensor([70, 50], dtype=torch.int32, device="cuda"))
    qx = torch.tensor([-5, 40, 1 << 30], dtype=torch.int32, device="cuda")
    kx = torch.tensor([-(1 << 31), 70, 121], dtype=torch.int32, device="cuda")
    kl = torch.tensor([71, 1 << 30], dtype=torch.int32, device="cuda")
    got = ops.attention_forward(q, k, v, qx, kx, k_lengths=kl)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    dout = rand(gen(102), *q.shape, dtype=BF)
    for a, b in zip(ops.attention_backward(dout, q, k, v, *got, qx, kx, k_lengths=kl), ops.attention_backward(dout, q, k, v, *want, qo, ko)):
        assert torch.equal(a, b)
    kl = torch.tensor([-3, 0], dtype=torch.int32, device="cuda")
    got = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl)
    assert (got[0] == 0).all() and (got[1] == -INF).all()


def test_refused_tensors_of_these(ops):  # noqa: F811
    q, k, v, qo, ko, kl = make(111, [4, 4], [6, 6], 4, 2, 8, BF, room=2)
    out, lse = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl)
    x, pos, f = q, torch.zeros(8, dtype=torch.int64, device="cuda"), ops.rotary_frequencies(8)
    m, seed = torch.zeros(4, 8, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda")
    A, B, R, D = ops.attention_forward, ops.attention_backward, ops.rotary_forward, ops.dropout_forward
    for call in (
            lambda: A(q.float(), k.float(), v.float(), qo, ko), lambda: A(q, k.half(), v, qo, ko), lambda: A(q, k, v[:-1], qo, ko),
            lambda: A(q, k[:, :, :7], v, qo, ko), lambda: A(q[:, :3], k, v, qo, ko), lambda: A(q[0], k, v, qo, ko),
            lambda: A(q, k, v, qo[:2], ko), lambda: A(q, k, v, qo, ko.long()), lambda: A(q, k, v, qo.float(), ko), lambda: A(q, k, v, qo[:1], ko[:1]),
            lambda: A(q, k, v, qo, ko, k_lengths=kl[:1]), lambda: A(q, k, v, qo, ko, k_lengths=kl.long()), lambda: A(q, k, v, qo.cpu(), ko),
            lambda: A(q, k.cpu(), v, qo, ko), lambda: A(q, k, v, qo, ko, scale=0.0), lambda: A(q, k, v, qo, ko, scale=-1.0),
            lambda: A(q.transpose(1, 2), k, v, qo, ko), lambda: A(q[:, :1].expand(8, 4, 8), k, v, qo, ko), lambda: A(q[:1].expand(8, 4, 8), k, v, qo, ko),
            lambda: A(q[..., :0], k[..., :0], v[..., :0], qo, ko),
            lambda: B(out[:7], q, k, v, out, lse, qo, ko), lambda: B(out, q, k, v, out.half(), lse, qo, ko), lambda: B(out, q, k, v, out, lse.t(), qo, ko),
            lambda: B(out, q, k, v, out, lse.double(), qo, ko), lambda: B(out, q, k, v, out, lse[:, ::2], qo, ko),
            lambda: R(x, pos[:7], f), lambda: R(x, pos.float(), f), lambda: R(x, pos, f.float()), lambda: R(x, pos, f[:0]), lambda: R(x, pos, f[None]),
            lambda: R(x, pos, ops.rotary_frequencies(10)), lambda: R(x.double(), pos, f), lambda: R(x[0], pos, f), lambda: R(x, pos, f, out=x.half()),
            lambda: R(x, pos, f, out=x[:7]), lambda: R(x, pos.cpu(), f),
            lambda: D(m, -0.1, seed), lambda: D(m, 1.5, seed), lambda: D(m, float("nan"), seed), lambda: D(m, 0.1, seed[:1]), lambda: D(m, 0.1, seed.int()),
            lambda: D(m, 0.1, seed.cpu()), lambda: D(m, 0.1, seed, residual=m.half()), lambda: D(m, 0.1, seed, residual=m[:3]), lambda: D(m[0], 0.1, seed),
            lambda: D(m.t(), 0.1, seed)):
        assert refused(ops, call)
    from paper_2407_04001_amd import PaseError
    wide = torch.zeros(2, 1, 136, dtype=BF, device="cuda")
    with pytest.raises(PaseError) as e:
        A(wide, wide, wide, offsets([2]), offsets([2]))
    assert e.value.status == 5   # too large


def test_nothing_to_attend(ops):  # noqa: F811
    """No rows, no keys, no heads' worth of either: outputs of 0."""
    z = torch.zeros(0, 2, 16, dtype=BF, device="cuda")
    q = rand(gen(121), 5, 4, 16, dtype=BF)
    none, five = offsets([0]), offsets([5])
    out, lse = ops.attention_forward(q, z, z, five, none)
    assert (out == 0).all() and (lse == -INF).all()
    dq, dk, dv = ops.attention_backward(q, q, z, z, out, lse, five, none)
    assert (dq == 0).all() and dk.shape == (0, 2, 16)
    zq, k = z.new_empty(0, 4, 16), rand(gen(122), 7, 2, 16, dtype=BF)
    out, lse = ops.attention_forward(zq, k, k, none, offsets([7]))
    assert out.shape == (0, 4, 16) and lse.shape == (4, 0)
    dq, dk, dv = ops.attention_backward(zq, zq, k, k, out, lse, none, offsets([7]))
    assert dq.shape == (0, 4, 16) and (dk == 0).all() and (dv == 0).all()
    empty = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert ops.rotary_forward(zq, empty, ops.rotary_frequencies(16)).shape == (0, 4, 16)
    assert ops.dropout_forward(torch.zeros(0, 9, device="cuda"), 0.5, torch.zeros(2, dtype=torch.int64, device="cuda")).shape == (0, 9)


def test_differentiable_forms(ops):  # noqa: F811
    """Gradients through autograd are the passes' own, also for expanded and strided gradients, and second ones are refused."""
    q, k, v, qo, ko, kl = make(131, [20, 30], [25, 35], 4, 2, 32, HF, room=7)
    k, v = k.nan_to_num(0.0), v.nan_to_num(0.0)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out = ops.attention(*leaves, qo, ko, k_lengths=kl, causal=True, scale=0.3)
    want, lse = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=True, scale=0.3)
    assert torch.equal(out, want)
    for dout in (rand(gen(1), *q.shape, dtype=HF), torch.ones((), dtype=HF, device="cuda").expand(q.shape), rand(gen(2), 32, 4, 50, dtype=HF).permute(2, 1, 0)):
        got = torch.autograd.grad(out, leaves, dout, retain_graph=True)
        ref = ops.attention_backward(dout.contiguous(), q, k, v, want, lse, qo, ko, k_lengths=kl, causal=True, scale=0.3)
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    f, pos = ops.rotary_frequencies(32), torch.arange(50, device="cuda")
    x = q.clone().requires_grad_()
    y = ops.rotary(x, pos, f, interleaved=True, magnitude=1.5)
    dy = torch.ones((), dtype=HF, device="cuda").expand(q.shape)
    assert torch.equal(torch.autograd.grad(y, x, dy, retain_graph=True)[0], ops.rotary_backward(dy.contiguous(), pos, f, interleaved=True, magnitude=1.5))
    seed = torch.tensor([1, 2], device="cuda")
    m, r = rand(gen(3), 50, 33).requires_grad_(), rand(gen(4), 50, 33).requires_grad_()
    z = ops.dropout(m, 0.3, seed, residual=r)
    seed.add_(1)   # the backward pass takes the seed that the forward pass had
    dm, dr = torch.autograd.grad(z, (m, r), torch.ones((), device="cuda").expand(50, 33), retain_graph=True)
    assert torch.equal(dr, torch.ones_like(r)) and torch.equal(dm, ops.dropout_backward(torch.ones(50, 33, device="cuda"), 0.3, torch.tensor([1, 2], device="cuda")))
    for out, leaf in ((ops.attention(*leaves, qo, ko, k_lengths=kl), leaves[0]), (ops.rotary(x, pos, f), x), (ops.dropout(m, 0.3, seed), m)):
        grad, = torch.autograd.grad(out.square().sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError):
            grad.sum().backward()


def test_rotation_in_place_is_known_to_autograd(ops):  # noqa: F811
    x = rand(gen(141), 6, 2, 8).requires_grad_()
    h = x * 2
    y = h.square().sum()   # saved h
    ops.rotary_forward(h.detach(), torch.arange(6, device="cuda"), ops.rotary_frequencies(8), out=h.detach())
    with pytest.raises(RuntimeError):
        y.backward()


def test_outputs_keep_to_their_rows_and_heads(ops):  # noqa: F811
    """Through the C ABI with wider outputs: what lies between heads and rows is untouched."""
    L = ops.load()
    q, k, v, qo, ko, _ = make(151, [70, 30], [50, 61], 4, 2, 40, BF)
    rows, keys, mark = q.shape[0], k.shape[0], 7.5
    stream = torch.cuda.current_stream().cuda_stream

    def room(rows, heads):
        return torch.full((rows + 2, heads + 1, 43), mark, dtype=BF, device="cuda")

    def inside(t):
        return t[1:-1, :-1, :40]

    def untouched(t):
        u = t.clone()
        inside(u)[:] = mark
        return bool((u == mark).all())

    def arg(t):
        return t.data_ptr(), t.stride(0), t.stride(1)

    out, lse = room(rows, 4), torch.empty(4, rows, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    ref = ops.attention_forward(q, k, v, qo, ko, causal=True)
    assert L.pase_attention_forward(0, rows, keys, 2, 4, 2, 40, *arg(q), *arg(k), *arg(v), qo.data_ptr(), ko.data_ptr(), None, 0, 1, 40 ** -0.5,
                                    *arg(inside(out)), lse.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0
    assert torch.equal(inside(out), ref[0]) and torch.equal(lse, ref[1]) and untouched(out)
    dq, dk, dv = room(rows, 4), room(keys, 2), room(keys, 2)
    assert L.pase_attention_backward(0, rows, keys, 2, 4, 2, 40, *arg(q), *arg(q), *arg(k), *arg(v), *arg(inside(out)), lse.data_ptr(), qo.data_ptr(),
                                     ko.data_ptr(), None, 0, 1, 40 ** -0.5, *arg(inside(dq)), *arg(inside(dk)), *arg(inside(dv)), ws.data_ptr(), ws.numel(), stream) == 0
    for t, want in zip((dq, dk, dv), ops.attention_backward(q, q, k, v, *ref, qo, ko, causal=True)):
        assert torch.equal(inside(t), want) and untouched(t)
    y, pos, f = room(rows, 4), torch.arange(rows, device="cuda"), ops.rotary_frequencies(24)
    assert L.pase_rotary(0, rows, 4, 40, 24, 1, 0, *arg(q), pos.data_ptr(), 1, f.data_ptr(), 1.0, *arg(inside(y)), stream) == 0
    assert torch.equal(inside(y), ops.rotary_forward(q, pos, f, interleaved=True)) and untouched(y)
    m, z, seed = rand(gen(9), rows, 40, dtype=BF), torch.full((rows, 43), mark, dtype=BF, device="cuda"), torch.tensor([3, 4], device="cuda")
    assert L.pase_dropout(0, rows, 40, m.data_ptr(), 40, None, 0, 0.5, seed.data_ptr(), z.data_ptr(), 43, stream) == 0
    assert torch.equal(z[:, :40], ops.dropout_forward(m, 0.5, seed)) and (z[:, 40:] == mark).all()


def test_attention_of_more_tiles_than_one_launch_holds(ops):  # noqa: F811
    """65536 sequences of one token and one key under 256 heads: over 2^24 workgroups of 256 threads in every kernel.
    A weight of 1 makes the output the value and dv the gradient, both exactly; ds is what two orders of one sum leave."""
    n, heads, dim = 65536, 256, 8
    g = gen(161)
    q, k, v, dout = (rand(g, n, heads, dim, dtype=BF) for _ in range(4))
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out, lse = ops.attention_forward(q, k, v, off, off, causal=True)
    assert torch.equal(out, v)
    want = (q.double() * k.double()).sum(2).t() * dim ** -0.5
    size = (q.double() * k.double()).abs().sum(2).t() * dim ** -0.5
    assert ((lse.double() - want).abs() <= 2 * (dim + 8) * E * size + 8 * E * want.abs() + 2.0 ** -21).all()
    dq, dk, dv = ops.attention_backward(dout, q, k, v, out, lse, off, off, causal=True)
    # p = exp(s - lse) is 1 but for the roundings of s, lse and the power
    p_error = (4 * (dim + 8) * E * size + 16 * E * want.abs() + 2.0 ** -20).t()[..., None]
    assert ((dv.double() - dout.double()).abs() <= (U[BF] + p_error) * dout.double().abs()).all()
    noise = (4 * (dim + 8) * E * (dout.double() * v.double()).abs().sum(2))[..., None]
    assert (dq.double().abs() <= 1.1 * dim ** -0.5 * noise * k.double().abs()).all()
    assert (dk.double().abs() <= 1.1 * dim ** -0.5 * noise * q.double().abs()).all()


def test_rotary_of_more_rows_than_one_launch_holds(ops):  # noqa: F811
    x = torch.zeros((1 << 24) + 5, 1, 258, dtype=BF, device="cuda")
    x[-3:] = rand(gen(171), 3, 1, 258, dtype=BF)
    positions = torch.arange(x.shape[0], device="cuda")
    f = ops.rotary_frequencies(258)
    want = ops.rotary_forward(x[-3:].contiguous(), positions[-3:], f)
    ops.rotary_forward(x, positions, f, out=x)
    assert torch.equal(x[-3:], want) and not x[:-3].any()
