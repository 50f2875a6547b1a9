"""Attention, rotary positions and dropout where calls that the documentation allows come close to its limits.

Tolerances are the bounds of test_attention_gpu: u is the unit roundoff of a matrix's type, e = 2^-24 that of fp32."""
import math

import pytest
import torch

from test_attention_gpu import bounds, check_backward, check_forward, laid_out, make, offsets, rotary64, sequences  # noqa: F401
from test_operators_gpu import BF, E, HF, INF, SF, U, close, gen, ops, rand, refused  # noqa: F401

pytestmark = pytest.mark.gpu


def arg(t, ld=None):
    """Pointer and strides of a [rows, heads, dim] argument of the C ABI."""
    return t.data_ptr(), t.stride(0) if ld is None else ld, t.stride(1)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [24, 64, 126, 128, 13])
@pytest.mark.parametrize("keys,heads,kv_heads", [(70, 4, 2), (1, 3, 3), (700, 2, 1)])
def test_one_row_has_no_row_stride(ops, keys, heads, kv_heads, dim, dtype):  # noqa: F811
    """Through the C ABI: the row stride of a single row, whatever it is, has no influence."""
    L = ops.load()
    g = gen(201)
    q, dout, out2 = (rand(g, 1, heads, dim, dtype=dtype) for _ in range(3))
    k, v = rand(g, keys, kv_heads, dim, dtype=dtype), rand(g, keys, kv_heads, dim, dtype=dtype)
    qo, ko = offsets([1]), offsets([keys])
    ref = ops.attention_forward(q, k, v, qo, ko)
    grads = ops.attention_backward(dout, q, k, v, *ref, qo, ko)
    check_backward(grads, dout, q, k, v, *ref, qo, ko)
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    stream, code = torch.cuda.current_stream().cuda_stream, 0 if dtype is BF else 1
    for ld in (0, 1, dim // 2, dim - 1):
        key_ld = ld if keys == 1 else None
        lse, dq, dk, dv = (torch.full_like(t, float("nan")) for t in (ref[1], q, k, v))
        assert L.pase_attention_forward(code, 1, keys, 1, heads, kv_heads, dim, *arg(q, ld), *arg(k, key_ld), *arg(v, key_ld), qo.data_ptr(),
                                        ko.data_ptr(), None, 0, 0, dim ** -0.5, *arg(out2, ld), lse.data_ptr(), ws.data_ptr(), ws.numel(), stream) == 0
        assert torch.equal(out2, ref[0]) and torch.equal(lse, ref[1]), ld
        assert L.pase_attention_backward(code, 1, keys, 1, heads, kv_heads, dim, *arg(dout, ld), *arg(q, ld), *arg(k, key_ld), *arg(v, key_ld),
                                         *arg(out2, ld), lse.data_ptr(), qo.data_ptr(), ko.data_ptr(), None, 0, 0, dim ** -0.5, *arg(dq, ld),
                                         *arg(dk, key_ld), *arg(dv, key_ld), ws.data_ptr(), ws.numel(), stream) == 0
        for name, a, b in zip(("dq", "dk", "dv"), (dq, dk, dv), grads):
            assert torch.equal(a, b), (name, ld)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_many_small_weights_count(ops, dtype):  # noqa: F811
    """A key far above the others, whose weights e^-18 are below half of fp16's least number: together they are 0.2 % of the
    output.  Half the spacing of fp16's subnormals is 2^-25, of weights that are 2^6 times their size 2^-31 for each."""
    rows, keys, heads, dim = 8192, 131072, 4, 32   # 256 tiles of 128 queries
    q, k, v = (torch.zeros(n, heads, dim, dtype=dtype, device="cuda") for n in (rows, keys, keys))
    q[..., 0], k[0, :, 0], v[1:] = 4.5, 4.0, 1.0
    out, lse = ops.attention_forward(q, k, v, offsets([rows]), offsets([keys]), scale=1.0)
    rest = (keys - 1) * math.exp(-18)
    want = rest / (1 + rest)
    error = 2 * (dim + 8) * E * 18 + 8 * E * 18 + 2.0 ** -21   # of a weight, as in the bounds of test_attention_gpu
    tol = want * (2 * U[dtype] + 2 * error + 4 * (keys + 8) * E) + (keys * 2.0 ** -31 if dtype is HF else 0.0)
    assert (out.double() - want).abs().max() <= tol
    assert (lse.double() - (18 + math.log1p(rest))).abs().max() <= error + (keys + 8) * E + 8 * E * 18


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,keys,far", [(4096, 256, True), (128, 166937, False), (2048, 166937, False)])
def test_gradients_of_many_small_weights(ops, rows, keys, far, dtype):  # noqa: F811
    """dv of weights that are 2^-26, or 100.5 times fp16's least number: each is rounded by u of itself all the same."""
    dim = 32
    q, k, v = (torch.zeros(n, 1, dim, dtype=dtype, device="cuda") for n in (rows, keys, keys))
    if far:
        q[..., 0], k[0, :, 0] = 4.5, 4.0
    dout = torch.full_like(q, 16.0)
    qo, ko = offsets([rows]), offsets([keys])
    out, lse = ops.attention_forward(q, k, v, qo, ko, scale=1.0)
    dq, dk, dv = ops.attention_backward(dout, q, k, v, out, lse, qo, ko, scale=1.0)
    top = 18.0 if far else 0.0
    l = top + math.log1p((keys - 1) * math.exp(-18)) if far else math.log(keys)
    want = rows * 16 * math.exp(-l)
    # (weights that are all alike are powers of two, and their sums below 2^24 of them exact)
    error = 2 * (dim + 8) * E * top + 16 * E * l + 2.0 ** -20 + ((keys + 8) * E if far else 0.0)
    assert (dv[1:].double() - want).abs().max() <= want * (2 * U[dtype] + 2 * error + 2 * (rows + 8) * E)
    assert (dq == 0).all() and (dk == 0).all()   # values of 0


def test_many_kept_keys_of_one_large_group(ops):  # noqa: F811
    """2^29 keys under 128 heads that share them: their rows x heads are within the limit."""
    keys, heads = 1 << 29, 128
    k, v = torch.zeros(keys, 1, 2, dtype=BF, device="cuda"), torch.ones(keys, 1, 2, dtype=BF, device="cuda")
    k[-1, 0, 0], v[-1] = 40.0, 3.0
    q = torch.zeros(1, heads, 2, dtype=BF, device="cuda")
    q[0, 64:, 0] = 1.0
    out, lse = ops.attention_forward(q, k, v, offsets([1]), torch.tensor([0, keys], dtype=torch.int32, device="cuda"), causal=True, scale=1.0)
    # half of the heads see all keys alike, the others the last one: e^40 against 2^29
    assert (out[0, :64] == 1).all() and (out[0, 64:] == 3).all()
    want = torch.tensor([29 * math.log(2)] * 64 + [40 + math.log1p((keys - 1) * math.exp(-40))], dtype=torch.double, device="cuda")
    got = lse[:65, 0].double()
    assert ((got - want).abs() <= 16 * E * want + 2.0 ** -20).all()
    assert (lse[65:, 0] == lse[64, 0]).all()


def test_out_that_overlaps_x_is_refused(ops):  # noqa: F811
    """rotary's out is x, or has no element of it."""
    f = ops.rotary_frequencies(8)
    b = rand(gen(211), 40, 6, 8, dtype=BF)
    kept, pos = b.clone(), torch.arange(20, device="cuda")
    x = b[:20, :4]
    for out in (b[1:21, :4], b[19:39, :4], b[:20, 1:5], b[:20, 2:6], b[1:21, 1:5]):
        assert refused(ops, lambda: ops.rotary_forward(x, pos, f, out=out))
        assert refused(ops, lambda: ops.rotary_backward(out, pos, f, out=x))
    flat = b.view(-1)
    assert refused(ops, lambda: ops.rotary_forward(x, pos, f, out=torch.as_strided(flat, (20, 4, 8), (48, 8, 1), 4)))
    assert torch.equal(b, kept)
    # no element in common: other rows, other heads of the same rows, the other half of wider heads
    for x, out in ((b[:20], b[20:]), (b[20:], b[:20]), (b[:20, :3], b[:20, 3:]), (b[:20, 4:], b[:20, 1:3]),
                   (torch.as_strided(flat, (20, 2, 8), (48, 16, 1), 0), torch.as_strided(flat, (20, 2, 8), (48, 16, 1), 8))):
        want = ops.rotary_forward(x, pos, f)
        assert ops.rotary_forward(x, pos, f, out=out) is out
        assert torch.equal(out, want)


def test_gradients_whose_rows_are_far_apart(ops):  # noqa: F811
    """Autograd may hand over a slice of a wide gradient, with rows further apart than the operators take."""
    q, k, v, qo, ko, _ = make(251, [20, 10], [25, 15], 4, 2, 16, BF)
    wide = torch.zeros(30, (1 << 22) + 64, dtype=BF, device="cuda")
    dout = wide[:, 64:128].view(30, 4, 16)
    dout.copy_(rand(gen(252), 30, 4, 16, dtype=BF))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out, lse = ops.attention_forward(q, k, v, qo, ko)
    got = torch.autograd.grad(ops.attention(*leaves, qo, ko), leaves, dout)
    assert all(torch.equal(a, b) for a, b in zip(got, ops.attention_backward(dout.contiguous(), q, k, v, out, lse, qo, ko)))
    f, pos = ops.rotary_frequencies(16), torch.arange(30, device="cuda")
    got, = torch.autograd.grad(ops.rotary(leaves[0], pos, f), leaves[0], dout)
    assert torch.equal(got, ops.rotary_backward(dout.contiguous(), pos, f))


# Offsets for which tiles of keys are dealt by place (four teams: at least 16 steps of the average sequence; keys of 16 tiles of 64 a
# sequence) with ranges in both halves of the search, that is 63 to 126 sequences.
BY_PLACE = [
    ([520] * 100 + [900], [1100] * 101, 2, 1, 32, {"room": 1}),
    ([520] * 62 + [530], [1030 + 37 * (i % 5) for i in range(63)], 1, 1, 64, {}),
    ([18 * (i % 62) for i in range(126)], [19 * ((i * 7) % 126) for i in range(126)], 1, 1, 64, {"before": 3, "after": 2}),
    ([0] * 80 + [412] + [0] * 20, [0] * 40 + [70] * 40 + [102000] + [1] * 20, 128, 1, 64, {}),
]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("case", BY_PLACE, ids=[f"{len(c[0])}_h{c[2]}-{c[3]}_d{c[4]}" for c in BY_PLACE])
def test_keys_of_many_long_sequences(ops, case, dtype):  # noqa: F811
    *sizes, rest = case
    n, group, step = len(sizes[0]), sizes[2] // sizes[3], 64 if sizes[4] == 32 else 32
    q, k, v, qo, ko, kl = make(221, *sizes, dtype, **rest)
    assert q.shape[0] // n * group // step >= 16 and 64 < n + 2 <= 128 and k.shape[0] >= 16 * 64 * n
    dout = rand(gen(222), *q.shape, dtype=dtype, scale=0.5)
    out, lse = ops.attention_forward(q, k, v, qo, ko, k_lengths=kl, causal=True)
    check_forward((out, lse), q, k, v, qo, ko, kl, True)
    check_backward(ops.attention_backward(dout, q, k, v, out, lse, qo, ko, k_lengths=kl, causal=True), dout, q, k, v, out, lse, qo, ko, kl, True)


@pytest.mark.parametrize("rows,keys,heads,kv_heads,q_offsets,k_offsets", [
    (100, 120, 4, 2, [0, 60, 40, 100], [0, 100, 30, 120]),             # one tile each
    (100, 120, 4, 2, [90, 50, 10, 0], [120, 80, 5, -7]),               # only decreasing
    (4, 9000, 4, 4, [0, 3, 1, 4], [0, 8000, 500, 9000]),               # few queries: shares and their join
    (3000, 3000, 4, 1, [0, 2500, 100, 3000], [0, 2900, 50, 3000]),     # four teams, dealt by place
    (40, 40, 2, 2, [40, 0] * 90, [0, 40] * 90),                        # more ranges than a wave has lanes
])
@pytest.mark.parametrize("dim", [64, 13])
def test_decreasing_offsets_keep_to_the_outputs(ops, rows, keys, heads, kv_heads, q_offsets, k_offsets, dim):  # noqa: F811
    """Results are undefined there, but nothing outside the outputs is written and the calls end."""
    L = ops.load()
    g = gen(231)
    n, mark = len(q_offsets) - 1, 7.5
    q, dout = rand(g, rows, heads, dim, dtype=BF), rand(g, rows, heads, dim, dtype=BF)
    k, v = rand(g, keys, kv_heads, dim, dtype=BF), rand(g, keys, kv_heads, dim, dtype=BF)
    qo, ko = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (q_offsets, k_offsets))
    stream = torch.cuda.current_stream().cuda_stream

    def room(rows, heads):
        return torch.full((rows + 2, heads + 1, dim + 1), mark, dtype=BF, device="cuda")

    def untouched(t):
        u = t.clone()
        u[1:-1, :-1, :dim] = mark
        return bool((u == mark).all())

    def guarded(n, dtype=torch.float32):
        return torch.full((n + 512,), mark, dtype=dtype, device="cuda")

    def place(t):
        return arg(t[1:-1, :-1, :dim])

    lse = guarded(heads * rows)
    for backward in (0, 1):
        need = ops._bytes("pase_attention_workspace", 0, rows, keys, n, heads, kv_heads, dim, backward)
        ws = guarded(need // 4)
        if not backward:
            out = room(rows, heads)
            assert L.pase_attention_forward(0, rows, keys, n, heads, kv_heads, dim, *arg(q), *arg(k), *arg(v), qo.data_ptr(), ko.data_ptr(), None, 0, 1,
                                            dim ** -0.5, *place(out), lse.data_ptr(), ws.data_ptr(), need, stream) == 0
            outs = [out]
        else:
            outs = [room(rows, heads), room(keys, kv_heads), room(keys, kv_heads)]
            assert L.pase_attention_backward(0, rows, keys, n, heads, kv_heads, dim, *arg(dout), *arg(q), *arg(k), *arg(v), *place(out), lse.data_ptr(),
                                             qo.data_ptr(), ko.data_ptr(), None, 0, 1, dim ** -0.5, *(a for t in outs for a in place(t)), ws.data_ptr(),
                                             need, stream) == 0
        assert all(untouched(t) for t in outs) and (lse[heads * rows:] == mark).all() and (ws[need // 4:] == mark).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_of_rotation_and_dropout_by_differences(ops, interleaved):  # noqa: F811
    """Against central differences of the 64-bit definitions along random directions; both are linear, so that the differences are
    exact but for 2^-53 of their terms over the step, and a gradient element is off by u of itself and its own fp32 steps."""
    g = gen(241)
    x, dy = rand(g, 9, 3, 26, dtype=HF), rand(g, 9, 3, 26, dtype=HF)
    f, pos = ops.rotary_frequencies(24), torch.arange(9, device="cuda") * 100
    seed = torch.tensor([7, 8], device="cuda")
    keep = ops.dropout_forward(torch.ones(27, 26, device="cuda"), 0.25, seed).view(9, 3, 26) != 0   # (test_dropout has the mask from its definition)
    for dx, value in ((ops.rotary_backward(dy, pos, f, interleaved=interleaved, magnitude=1.25), lambda t: rotary64(t, pos, f, interleaved, 1.25)),
                      (ops.dropout_backward(dy.view(27, 26), 0.25, seed).view(9, 3, 26), lambda t: torch.where(keep, t / 0.75, 0.0))):
        for _ in range(3):
            d = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.double)
            e = 2.0 ** -10
            slope = ((value(x.double() + e * d) - value(x.double() - e * d)) * dy.double()).sum() / (2 * e)
            # the rotation's terms are at most 1.25 (|a| + |b|)
            size = (2 * 1.25 * dy.double().abs().amax() * d.abs()).sum()
            assert (slope - (dx.double() * d).sum()).abs() <= (U[HF] + 16 * E) * (dx.double().abs() * d.abs()).sum() + 2.0 ** -20 * size


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows,far", [(8192, 18.0), (8192, 16.5), (1, 16.5)])
def test_long_sums_behind_a_large_weight(ops, rows, far, dtype):  # noqa: F811
    """The weights' sum after a first one of 1: 131071 of e^-18 or e^-16.5, each below half of the last bit of 1.  A lane adds up its weights
    of a step of keys, at most 32 of the 64, then the steps: these sums are off by E each, of less than 2."""
    keys, heads, dim = 131072, 4, 32
    q, k, v = (torch.zeros(n, heads, dim, dtype=dtype, device="cuda") for n in (rows, keys, keys))
    q[..., 0], k[0, :, 0], v[:] = 1.0, far, 1.0
    out, lse = ops.attention_forward(q, k, v, offsets([rows]), offsets([keys]), scale=1.0)
    want = far + math.log1p((keys - 1) * math.exp(-far))
    weight = 2 * (dim + 8) * E * far + 8 * E * far + 2.0 ** -21
    sums = (2 * keys / 64 + 64) * E
    assert (lse.double() - want).abs().max() <= weight * (keys - 1) * math.exp(-far) + 2.0 ** -21 + sums + 8 * E * far
    # values of 1: the products' sum is rounded in other places, over 16 keys at a time
    assert (out.double() - 1).abs().max() <= U[dtype] * 2 + sums + 2 * (keys / 16 + 16) * E * 2 + (keys * 2.0 ** -31 if dtype is HF else 0)
