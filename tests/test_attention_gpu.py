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
