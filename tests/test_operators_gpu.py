"""The layer operators on the GPU against their definitions in 64 bits.

Tolerances are bounds, not fits.  With u the unit roundoff of the output's type
and e = 2^-24 that of fp32, a sum of n fp32 terms in any order is off by at most
n e times the sum of their magnitudes (twice that where the matrix unit may
truncate), and every result is rounded once, by at most u of itself.  Products
of small whole numbers have exact sums and are compared for equality."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float32: 0.0}   # half the spacing of subnormals
BF, HF, SF = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def ops():
    from paper_2407_04001_amd import ops as O
    O.load()
    return O


def rand(gen, *shape, dtype=SF, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(dtype)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def wide(t, pad, fill=float("nan")):
    """t as a column slice of a wider buffer that holds NaN elsewhere."""
    if not pad:
        return t
    b = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=t.device)
    b[:, :t.shape[1]] = t
    return b[:, :t.shape[1]]


def close(got, want, tol, what=""):
    """|got - want| <= tol + the rounding to got's type, elementwise; NaN and infinities alike."""
    w = want.double()
    same = (got.double() == w) | (got.double().isnan() & w.isnan())
    bound = tol + (U[got.dtype] * 1.01) * w.abs() + TINY[got.dtype]
    off = (got.double() - w).abs()
    ok = same | (off <= bound)
    assert ok.all(), f"{what}: {(~ok).sum()} of {ok.numel()} off, worst {(off / bound).nan_to_num(0, INF, 0)[~ok].max()} of its bound"


# ------------------------------------------------------------------ layer norm
def norm64(x, gain, bias, residual, eps):
    z = x.double() + (residual.double() if residual is not None else 0.0)
    mean = z.mean(1)
    rstd = 1 / ((z - mean[:, None]).square().mean(1) + eps).sqrt()
    h = (z - mean[:, None]) * rstd[:, None]
    y = h * gain.double() + (bias.double() if bias is not None else 0.0)
    return y, z, mean, rstd


def check_norm_forward(got, x, gain, bias, residual, eps):
    y, z, mean, rstd = norm64(x, gain, bias, residual, eps)
    gy, gz, gm, gr = got
    n = (x.shape[1] + 8) * E                       # of a row sum
    zerr = E * z.abs()                             # of the fp32 sum x + residual
    merr = n * z.abs().mean(1) + zerr.max(1).values
    # rstd = (v + eps)^-1/2: half the relative error of v, which sums squares of deviations off by merr + zerr
    dev = (z - mean[:, None]).abs()
    verr = (2 * dev * (merr[:, None] + zerr)).mean(1) + (merr + zerr.max(1).values) ** 2 + n * dev.square().mean(1)
    rerr = 0.5 * verr * rstd ** 3 * 1.5 + 4 * E * rstd
    close(gm, mean, merr, "mean")
    close(gr, rstd, rerr, "rstd")
    if residual is not None:
        close(gz, z, zerr, "z")
    tol = gain.double().abs() * (rstd[:, None] * (merr[:, None] + zerr + 2 * E * dev) + dev * rerr[:, None]) + 4 * E * y.abs() \
        + 2 * E * (bias.double().abs() if bias is not None else 0.0)
    close(gy, y, tol, "y")


NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (1, 8), (2, 63), (64, 64), (7, 65), (33, 342), (130, 511), (9, 512), (6, 513),
               (300, 1024), (31, 1025), (17, 2048), (4, 2049), (5, 4097), (3, 8192), (2, 8193), (3, 16384), (2, 16383)]


@pytest.mark.parametrize("dtype,param", [(BF, BF), (BF, SF), (HF, HF), (HF, SF), (SF, SF)])
@pytest.mark.parametrize("rows,width", NORM_SHAPES)
def test_norm_forward(ops, rows, width, dtype, param):
    g = gen(rows * 31 + width)
    x = wide(rand(g, rows, width, dtype=dtype, scale=2.0, shift=0.7), 3 if width % 2 else 0)
    res = wide(rand(g, rows, width, dtype=dtype), 8 if rows % 2 else 0)
    gain, bias = rand(g, width, dtype=param, scale=0.3, shift=1.0), rand(g, width, dtype=param)
    for r, b in ((res, bias), (None, bias), (res, None)):
        check_norm_forward(ops.layer_norm_forward(x, gain, b, residual=r, eps=1e-5), x, gain, b, r, 1e-5)


def norm_grad64(dy, z, gain, mean, rstd, dz):
    dy, z = dy.double(), z.double()
    h = (z - mean.double()[:, None]) * rstd.double()[:, None]
    dh = dy * gain.double()
    dx = rstd.double()[:, None] * (dh - dh.mean(1, keepdim=True) - h * (dh * h).mean(1, keepdim=True))
    if dz is not None:
        dx = dx + dz.double()
    return dx, (dy * h).sum(0), dy.sum(0), h, dh


def check_norm_backward(got, dy, z, gain, mean, rstd, dz):
    dx, dg, db, h, dh = norm_grad64(dy, z, gain, mean, rstd, dz)
    rows, width = dy.shape
    n, r = (width + 8) * E, rstd.double()[:, None]
    herr = 4 * E * (h.abs() + mean.double().abs()[:, None] * r)
    m0 = n * dh.abs().mean(1, keepdim=True)
    m1 = n * (dh * h).abs().mean(1, keepdim=True) + (dh.abs() * herr).mean(1, keepdim=True)
    mm = (dh * h).mean(1, keepdim=True).abs()
    tol = r * (m0 + h.abs() * m1 + herr * mm + 6 * E * (dh.abs() + dh.mean(1, keepdim=True).abs() + h.abs() * mm)) + 2 * E * dx.abs()
    if dz is not None:
        tol = tol + E * dz.double().abs()
    close(got[0], dx, tol, "dx")
    s = (rows + 8) * E
    close(got[1], dg, s * (dy.double() * h).abs().sum(0) + (dy.double().abs() * herr).sum(0), "dgain")
    close(got[2], db, s * dy.double().abs().sum(0), "dbias")


@pytest.mark.parametrize("dtype,param", [(BF, BF), (BF, SF), (HF, HF), (HF, SF), (SF, SF)])
@pytest.mark.parametrize("rows,width", NORM_SHAPES + [(2500, 320), (5000, 8)])
def test_norm_backward(ops, rows, width, dtype, param):
    g = gen(rows * 17 + width)
    dy = wide(rand(g, rows, width, dtype=dtype), 5 if width % 2 else 0)
    z = wide(rand(g, rows, width, dtype=dtype, scale=1.5, shift=-0.4), 8 if rows % 2 else 0)
    dz = rand(g, rows, width, dtype=dtype)
    gain = rand(g, width, dtype=param, scale=0.3, shift=1.0)
    _, _, mean, rstd = norm64(z, gain, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    for d in (dz, None):
        check_norm_backward(ops.layer_norm_backward(dy, z, gain, mean, rstd, dz=d), dy, z, gain, mean, rstd, d)


def test_norm_constant_and_extreme_rows(ops):
    """A constant row has variance 0; infinities and NaN stay in their row."""
    x = torch.randn(6, 300, device="cuda")
    x[1] = 3.25
    x[2, 7] = INF
    x[3, 299] = float("nan")
    x[4] = 1e30   # its squares overflow; its deviations are 0
    gain, bias = torch.rand(300, device="cuda") + 0.5, torch.randn(300, device="cuda")
    y, _, mean, rstd = ops.layer_norm_forward(x, gain, bias, eps=1e-5)
    assert torch.equal(y[1], bias) and mean[1] == 3.25
    assert y[2].isnan().all() and y[3].isnan().all()
    assert torch.isfinite(y[[0, 1, 5]]).all()
    keep = [0, 5]
    check_norm_forward(tuple(t[keep] for t in (y, x, mean, rstd)), x[keep], gain, bias, None, 1e-5)


def test_norm_large_mean(ops):
    """The variance of a row whose mean is 1000 deviations away."""
    g = gen(5)
    x = rand(g, 40, 1024, shift=1000.0)
    gain = torch.ones(1024, device="cuda")
    check_norm_forward(ops.layer_norm_forward(x, gain, eps=0.0), x, gain, None, None, 0.0)


def test_norm_no_rows(ops):
    x, gain = torch.zeros(0, 24, device="cuda"), torch.ones(24, device="cuda")
    y, z, mean, rstd = ops.layer_norm_forward(x, gain)
    assert y.shape == (0, 24) and mean.shape == (0,)
    dx, dg, db = ops.layer_norm_backward(x, x, gain, mean, rstd)
    assert dx.shape == (0, 24) and not dg.any() and not db.any()


def test_norm_gradient_by_differences(ops):
    """sum(y c) + sum(z d) of the definition in 64 bits, moved both ways along x, gain and bias."""
    g = gen(11)
    rows, width, eps, step = 5, 37, 1e-5, 1e-6
    x, res, c, d = (rand(g, rows, width) for _ in range(4))
    gain, bias = rand(g, width, shift=1.0), rand(g, width)
    y, z, mean, rstd = ops.layer_norm_forward(x, gain, bias, residual=res, eps=eps)
    dx, dg, db = ops.layer_norm_backward(c, z, gain, mean, rstd, dz=d)

    def f(x, gain, bias):
        y, z, _, _ = norm64(x, gain, bias, res, eps)
        return ((y * c.double()).sum() + (z * d.double()).sum()).item()

    for which, grad in enumerate((dx, dg, db)):
        for _ in range(3):
            v = rand(g, *grad.shape).double()
            at = [x.double(), gain.double(), bias.double()]
            up, down = list(at), list(at)
            up[which], down[which] = at[which] + step * v, at[which] - step * v
            slope = (f(*up) - f(*down)) / (2 * step)
            mine = (grad.double() * v).sum().item()
            # fp32 gradients of ~200 terms of size ~1 each (1e-5), differences in 64 bits (1e-7)
            assert abs(slope - mine) <= 1e-4 * (1 + grad.double().mul(v).abs().sum().item())


# ------------------------------------------------------------------ grouped products
def spans(offsets, rows):
    o = [min(max(int(v), 0), rows) for v in offsets.tolist()]
    return [(e, a, b) for e, (a, b) in enumerate(zip(o, o[1:])) if b > a]


def product64(x, w, offsets):
    y = torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64, device=x.device)
    mag = torch.zeros_like(y)
    for e, a, b in spans(offsets, x.shape[0]):
        we = w[e].double().t().contiguous()
        y[a:b] = x[a:b].double() @ we
        mag[a:b] = x[a:b].double().abs() @ we.abs()
    return y, mag


def product_grad64(dy, x, w, offsets):
    rows = x.shape[0]
    dx = torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    dw = torch.zeros(w.shape, dtype=torch.float64, device=x.device)
    mx, mw = torch.zeros_like(dx), torch.zeros_like(dw)
    for e, a, b in spans(offsets, rows):
        d, xe, we = dy[a:b].double(), x[a:b].double(), w[e].double()
        dx[a:b], mx[a:b] = d @ we, d.abs() @ we.abs()
        dt = d.t().contiguous()
        dw[e], mw[e] = dt @ xe, dt.abs() @ xe.abs()
    return dx, dw, mx, mw


def whole(g, *shape, dtype):
    """Whole numbers in -2 .. 2: products and sums of up to 2^22 of them are exact in fp32."""
    return torch.randint(-2, 3, shape, generator=g, device="cuda").to(dtype)


def ranges(lengths, lead=0, dtype=torch.int32):
    o = torch.tensor([lead] + lengths, dtype=torch.int64).cumsum(0)
    return o.to(dtype).cuda()


# lengths of the groups, rows before the first, rows after the last, n, k
PRODUCTS = [
    ([1], 0, 0, 1, 1), ([1], 0, 0, 8, 8), ([1], 0, 0, 1024, 512), ([3, 0, 1], 0, 0, 40, 24), ([0, 0], 0, 5, 16, 16),
    ([5, 9, 0, 31], 2, 3, 64, 64), ([16, 16], 0, 0, 128, 96), ([64] * 4, 0, 0, 65, 72), ([17, 33, 129], 0, 0, 127, 63),
    ([128, 128], 0, 0, 128, 128), ([200, 1, 57], 7, 0, 136, 200), ([300], 0, 0, 513, 130), ([256, 255, 257], 0, 1, 256, 264),
    ([700, 20], 0, 0, 300, 1366), ([1000, 24, 0, 1], 0, 100, 1366, 342), ([513], 0, 0, 1024, 1025),
    ([2] * 70, 1, 1, 48, 56), ([0] * 65 + [40], 0, 0, 32, 8), ([1] * 130, 0, 0, 24, 104), ([2100, 1500], 0, 0, 512, 768),
    ([4096, 13, 4000], 0, 0, 776, 520), ([12000], 0, 0, 264, 200), ([9, 7], 0, 0, 4096, 2048), ([3000, 2000, 1000], 0, 0, 2056, 1032),
]
PRODUCT_IDS = ["x".join(map(str, (len(p[0]), sum(p[0]) + p[1] + p[2], p[3], p[4]))) for p in PRODUCTS]


@pytest.mark.parametrize("case", PRODUCTS, ids=PRODUCT_IDS)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_product_forward_exact(ops, case, dtype):
    lengths, lead, spare, n, k = case
    g = gen(n * 7 + k)
    rows = lead + sum(lengths) + spare
    for pad, off in ((0, torch.int32), (8, torch.int64), (3, torch.int32)):
        x, w = wide(whole(g, rows, k, dtype=dtype), pad), whole(g, len(lengths), n, k, dtype=dtype)
        offsets = ranges(lengths, lead, off)
        y, _ = product64(x, w, offsets)
        assert torch.equal(ops.grouped_matmul_forward(x, w, offsets, out_dtype=SF), y.float()), pad
        assert torch.equal(ops.grouped_matmul_forward(x, w, offsets), y.to(dtype)), pad


@pytest.mark.parametrize("case", PRODUCTS, ids=PRODUCT_IDS)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_product_backward_exact(ops, case, dtype):
    lengths, lead, spare, n, k = case
    g = gen(n * 5 + k)
    rows = lead + sum(lengths) + spare
    for pad, grad in ((0, SF), (8, dtype), (3, SF)):
        x, w = wide(whole(g, rows, k, dtype=dtype), pad), whole(g, len(lengths), n, k, dtype=dtype)
        dy = wide(whole(g, rows, n, dtype=dtype), pad)
        offsets = ranges(lengths, lead)
        dx, dw, _, _ = product_grad64(dy, x, w, offsets)
        gx, gw = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=grad)
        assert torch.equal(gx, dx.to(dtype)), pad
        assert torch.equal(gw, dw.to(grad)), pad
        only, none = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=grad, need_dw=False)
        assert none is None and torch.equal(only, gx)
        none, only = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=grad, need_dx=False)
        assert none is None and torch.equal(only, gw)


@pytest.mark.parametrize("case", PRODUCTS[8:], ids=PRODUCT_IDS[8:])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_product_against_64_bits(ops, case, dtype):
    lengths, lead, spare, n, k = case
    g = gen(n * 3 + k)
    rows = lead + sum(lengths) + spare
    x, dy = rand(g, rows, k, dtype=dtype), rand(g, rows, n, dtype=dtype, scale=0.1)
    w = rand(g, len(lengths), n, k, dtype=dtype, scale=k ** -0.5)
    offsets = ranges(lengths, lead)
    y, mag = product64(x, w, offsets)
    for out in (dtype, SF):
        close(ops.grouped_matmul_forward(x, w, offsets, out_dtype=out), y, 2 * (k + 8) * E * mag, "y")
    dx, dw, mx, mw = product_grad64(dy, x, w, offsets)
    for grad in (dtype, SF):
        gx, gw = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=grad)
        close(gx, dx, 2 * (n + 8) * E * mx, "dx")
        close(gw, dw, 2 * (max(lengths) + 8) * E * mw, "dw")


@pytest.mark.parametrize("n,k", [(512, 512), (264, 511), (1000, 520)])
@pytest.mark.parametrize("groups,around", [(80, 100), (150, 90), (70, 300)])
def test_product_many_groups_exact(ops, groups, around, n, k):
    """More groups than a wave has lanes, with enough rows for the tiled kernels."""
    g = gen(groups + n)
    lengths = torch.randint(0, 2 * around, (groups,), generator=g, device="cuda").tolist()
    lengths[3] = lengths[groups - 1] = 0
    rows = 5 + sum(lengths) + 9
    x, dy, w = whole(g, rows, k, dtype=BF), whole(g, rows, n, dtype=BF), whole(g, groups, n, k, dtype=BF)
    offsets = ranges(lengths, 5)
    y, _ = product64(x, w, offsets)
    assert torch.equal(ops.grouped_matmul_forward(x, w, offsets, out_dtype=SF), y.float())
    dx, dw, _, _ = product_grad64(dy, x, w, offsets)
    gx, gw = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=SF)
    assert torch.equal(gx, dx.to(BF)) and torch.equal(gw, dw.float())


def test_product_infinities_stay_in_their_rows(ops):
    """NaN and infinities of rows of other groups, of no group and past a row's end reach no other row."""
    g = gen(3)
    lengths, n, k = [70, 60, 130], 136, 100
    x, w, dy = whole(g, 270, k, dtype=BF), whole(g, 3, n, k, dtype=BF), whole(g, 270, n, dtype=BF)
    offsets = ranges(lengths, 3)
    for bad in (float("nan"), INF):
        xb, db = wide(x, 4, bad).clone().as_strided(x.shape, (k, 1)), dy.clone()
        xb = wide(x, 4, bad)
        rows = [0, 2, 70, 263, 269]      # none, none, group 0, none, none
        xb[rows] = bad
        db[rows] = bad
        y = ops.grouped_matmul_forward(xb, w, offsets)
        want, _ = product64(x, w, offsets)
        keep = [r for r in range(270) if r not in rows]
        assert torch.equal(y[keep], want.to(BF)[keep])
        assert not y[[0, 2, 263, 269]].any() and not torch.isfinite(y[70]).any()
        gx, gw = ops.grouped_matmul_backward(db, xb, w, offsets)
        dx, dw, _, _ = product_grad64(dy, x, w, offsets)
        assert torch.equal(gx[keep], dx.to(BF)[keep]) and not gx[[0, 2, 263, 269]].any()
        assert torch.equal(gw[1:], dw.to(BF)[1:]) and not torch.isfinite(gw[0]).any()


def test_product_offsets_out_of_rule(ops):
    """Offsets that decrease or leave 0 .. rows are clamped: rows that one group alone holds are right."""
    g = gen(4)
    x, w = whole(g, 50, 40, dtype=BF), whole(g, 3, 24, 40, dtype=BF)
    offsets = torch.tensor([-5, 20, 90, 7], dtype=torch.int64, device="cuda")
    y = ops.grouped_matmul_forward(x, w, offsets, out_dtype=SF)
    want, _ = product64(x, w, torch.tensor([0, 20, 50, 50]))
    assert torch.equal(y[:7], want.float()[:7])
    ops.grouped_matmul_backward(whole(g, 50, 24, dtype=BF), x, w, offsets)
    torch.cuda.synchronize()


def test_product_no_rows(ops):
    w = torch.ones(2, 8, 16, dtype=BF, device="cuda")
    x, dy = torch.zeros(0, 16, dtype=BF, device="cuda"), torch.zeros(0, 8, dtype=BF, device="cuda")
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert ops.grouped_matmul_forward(x, w, offsets).shape == (0, 8)
    dx, dw = ops.grouped_matmul_backward(dy, x, w, offsets)
    assert dx.shape == (0, 16) and not dw.any()


def test_product_gradient_by_differences(ops):
    g = gen(12)
    lengths, n, k = [3, 0, 6], 20, 12
    x, w, c = rand(g, 10, k, dtype=HF), rand(g, 3, n, k, dtype=HF), rand(g, 10, n, dtype=HF)
    offsets = ranges(lengths, 1)
    dx, dw = ops.grouped_matmul_backward(c, x, w, offsets, grad_dtype=SF)

    def f(x, w):
        return (product64(x, w, offsets)[0] * c.double()).sum().item()

    for which, grad in enumerate((dx, dw)):
        v = rand(g, *grad.shape).double()
        at = [x.double(), w.double()]
        up, down = list(at), list(at)
        up[which], down[which] = at[which] + 1e-4 * v, at[which] - 1e-4 * v
        slope = (f(*up) - f(*down)) / 2e-4
        # bilinear: the difference is exact but for 64-bit rounding; dx is rounded to half precision
        tol = U[grad.dtype] * (grad.double() * v).abs().sum().item() + 1e-5 * grad.double().abs().sum().item()
        assert abs(slope - (grad.double() * v).sum().item()) <= tol


def test_product_past_32_bits(ops):
    """Rows whose element offsets pass 2^31 and whose byte offsets pass 2^32."""
    rows, n, k = 1_200_000, 24, 2048
    w = whole(gen(1), 2, n, k, dtype=BF)
    x = torch.zeros(rows, k, dtype=BF, device="cuda")
    dy = torch.zeros(rows, n, dtype=BF, device="cuda")
    at = torch.tensor([0, 1_048_575, 1_048_576, 1_100_001, rows - 1], device="cuda")
    x[at], dy[at] = whole(gen(2), 5, k, dtype=BF), whole(gen(3), 5, n, dtype=BF)
    offsets = torch.tensor([0, 1_048_576, rows], dtype=torch.int64, device="cuda")
    y = ops.grouped_matmul_forward(x, w, offsets, out_dtype=SF)
    few = torch.tensor([0, 2, 5])
    want, _ = product64(x[at], w, few)
    assert torch.equal(y[at], want.float())
    assert torch.equal(y.abs().sum(1).nonzero()[:, 0], at[want.abs().sum(1) > 0])
    dx, dw, _, _ = product_grad64(dy[at], x[at], w, few)
    gx, gw = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=SF)
    assert torch.equal(gx[at], dx.to(BF)) and torch.equal(gw, dw.float())


# ------------------------------------------------------------------ softmax loss
def loss64(logits, targets, dloss, ignore=-100):
    """The definition, its rules for masked and ignored rows, and the bounds of the errors."""
    l = logits.double()
    rows, classes = l.shape
    one = torch.arange(rows, device=l.device)
    counts = targets != ignore
    known = counts & (targets >= 0) & (targets < classes)
    t = torch.where(known, targets, 0).long()
    lse = torch.logsumexp(l, 1)
    empty = lse == -INF
    loss = torch.where(empty, INF, lse - l[one, t])
    loss = torch.where(known, loss, float("nan"))
    p = torch.exp(l - torch.where(empty, 0.0, lse)[:, None])
    d = p.clone()
    d[one, t] -= 1
    g = dloss.double().expand(rows)[:, None]
    d = torch.where(empty[:, None], 0.0, d * g)
    d = torch.where(known[:, None], d, float("nan"))
    # exp of an fp32 difference: the difference's rounding, and 2 ulp of the result
    dist = torch.where(p > 0, (l - lse[:, None]).abs(), 0.0)
    rel = (dist + l.abs().nan_to_num(0, 0, 0) * (p > 0) + 4) * 2 * E
    serr = (p * rel).sum(1) + (classes + 8) * E + 2 * E
    lerr = serr + 4 * E * (lse.abs().nan_to_num(0, 0, 0) + 1)
    loss_err = lerr + 2 * E * (lse.abs() + l[one, t].abs()).nan_to_num(0, 0, 0)
    derr = (p * (rel + lerr[:, None] + 2 * E * lse.abs().nan_to_num(0, 0, 0)[:, None]) + 2 * E * (d / g).abs().nan_to_num(0, 0, 0)) * g.abs()
    zero = lambda v: torch.where(counts if v.dim() == 1 else counts[:, None], v, 0.0)  # noqa: E731
    return zero(loss), zero(lse), zero(d), zero(loss_err), zero(lerr), zero(derr)


def check_loss(ops, logits, targets, dloss, ignore=-100):
    loss, lse, d, el, es, ed = loss64(logits, targets, dloss, ignore)
    a, b = ops.softmax_loss_forward(logits, targets, ignore_index=ignore)
    close(a, loss, el, "loss")
    close(b, lse, es, "lse")
    c, s, g = ops.softmax_loss_grad(logits, targets, dloss, ignore_index=ignore)
    assert torch.equal(a.nan_to_num(1e9), c.nan_to_num(1e9)) and torch.equal(b.nan_to_num(1e9), s.nan_to_num(1e9))
    close(g, d, ed.nan_to_num(0, 0, 0), "dlogits, one pass")
    g2 = ops.softmax_loss_backward(dloss, logits, targets, b, ignore_index=ignore)
    close(g2, d, ed.nan_to_num(0, 0, 0), "dlogits")
    return g


LOSS_SHAPES = [(1, 1), (3, 2), (5, 7), (64, 64), (2, 511), (33, 512), (7, 1000), (300, 1025), (130, 2049), (1, 4096),
               (9, 8191), (40, 10923), (3, 32768), (260, 32768), (5, 32769), (1, 65536), (3, 131071), (2, 131073), (1, 262145)]


@pytest.mark.parametrize("dtype", [BF, HF, SF])
@pytest.mark.parametrize("rows,classes", LOSS_SHAPES)
def test_softmax_loss(ops, rows, classes, dtype):
    g = gen(rows + classes)
    logits = wide(rand(g, rows, classes, dtype=dtype, scale=3.0), 7 if rows % 2 else 0)
    targets = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    targets[torch.rand(rows, generator=g, device="cuda") < 0.2] = -100
    if rows % 2:
        targets = targets.int()
    check_loss(ops, logits, targets, rand(g, rows))
    check_loss(ops, logits, targets, torch.full((), 0.25, device="cuda"))


@pytest.mark.parametrize("classes", [5, 600, 5000, 40000, 140000])
@pytest.mark.parametrize("dtype", [BF, HF, SF])
def test_softmax_loss_masks(ops, classes, dtype):
    """Masked classes, masked targets, rows that are all masked, lowest values, ignored rows that hold NaN."""
    g = gen(classes)
    logits = rand(g, 12, classes, dtype=dtype, scale=2.0)
    targets = torch.randint(0, classes, (12,), generator=g, device="cuda")
    logits[0, 1:] = -INF                      # one class left, the target
    targets[0] = 0
    logits[1] = -INF                          # none left
    logits[2, classes // 2:] = -INF           # the target is masked
    targets[2] = classes - 1
    logits[3] = torch.finfo(dtype).min        # lowest value everywhere: uniform
    logits[4, 1:] = torch.finfo(dtype).min
    logits[5] = float("nan")                  # ignored
    targets[5] = -100
    logits[6, 0] = torch.finfo(dtype).max
    targets[7] = classes                      # out of range
    targets[8] = -1
    targets[9] = 2 ** 40
    logits[10, classes - 1] = float("nan")
    logits[11] = INF
    dloss = rand(g, 12)
    loss, lse = ops.softmax_loss_forward(logits, targets)
    keep = [0, 1, 2, 3, 4, 5, 6]
    check_loss(ops, logits[keep], targets[keep], dloss[keep])
    assert loss[[7, 8, 9, 10, 11]].isnan().all()
    assert loss[1] == INF and lse[1] == -INF and loss[2] == INF and loss[5] == 0 and lse[5] == 0
    for d in (ops.softmax_loss_grad(logits, targets, dloss)[2], ops.softmax_loss_backward(dloss, logits, targets, lse)):
        assert not d[1].any() and not d[5].any() and d[[7, 8, 9, 10, 11]].isnan().all()
        assert torch.isfinite(d[[0, 2, 3, 4, 6]]).all()


def test_softmax_loss_other_ignored_index(ops):
    g = gen(8)
    logits, targets = rand(g, 20, 30), torch.randint(0, 30, (20,), generator=g, device="cuda")
    targets[:5] = 3
    check_loss(ops, logits, targets, rand(g, 20), ignore=3)


@pytest.mark.parametrize("rows,classes", [(70, 300), (70, 40001), (3, 150000), (2, 300000)])
def test_softmax_loss_in_place(ops, rows, classes):
    g = gen(9)
    logits, targets = rand(g, rows, classes, dtype=BF), torch.randint(0, classes, (rows,), generator=g, device="cuda")
    dloss = torch.full((rows,), 1 / rows, device="cuda")
    want = ops.softmax_loss_grad(logits, targets, dloss)
    lse = want[1]
    a, b = logits.clone(), logits.clone()
    got = ops.softmax_loss_grad(a, targets, dloss, out=a)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and got[2] is a
    assert torch.equal(ops.softmax_loss_backward(dloss, b, targets, lse, out=b), ops.softmax_loss_backward(dloss, logits, targets, lse))


def test_softmax_loss_past_32_bits(ops):
    rows, classes = 70_000, 32_768
    logits = torch.zeros(rows, classes, dtype=BF, device="cuda")
    targets = torch.arange(rows, device="cuda") % classes
    at = [0, 65_535, 65_536, rows - 1]
    for r in at:
        logits[r, r % classes] = 4.0
    dloss = torch.ones((), device="cuda")
    loss, lse, d = ops.softmax_loss_grad(logits, targets, dloss, out=logits)
    flat, high = math.log(classes), math.log(classes - 1 + math.exp(4.0))
    assert abs(lse[1] - flat) < 1e-5 and abs(loss[1] - flat) < 1e-5
    for r in at:
        assert abs(lse[r] - high) < 1e-5 and abs(loss[r] - (high - 4)) < 1e-5
        assert abs(d[r, r % classes].item() - (math.exp(4 - high) - 1)) < 2 ** -8
        assert abs(d[r, (r + 1) % classes].item() / math.exp(-high) - 1) < 2 ** -8


def test_softmax_loss_no_rows(ops):
    logits, targets = torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, lse, d = ops.softmax_loss_grad(logits, targets, torch.zeros(0, device="cuda"))
    assert loss.shape == (0,) and d.shape == (0, 10)


def test_softmax_loss_gradient_by_differences(ops):
    g = gen(13)
    logits, targets, c = rand(g, 6, 50), torch.randint(0, 50, (6,), generator=g, device="cuda"), rand(g, 6)
    logits[2, 10:20] = -INF
    targets[2], targets[4] = 3, -100
    d = ops.softmax_loss_grad(logits, targets, c)[2].double()

    def f(l):
        return (loss64(l, targets, c)[0] * c.double()).sum().item()

    for _ in range(4):
        v = rand(g, 6, 50).double()
        slope = (f(logits.double() + 1e-6 * v) - f(logits.double() - 1e-6 * v)) / 2e-6
        assert abs(slope - (d * v).sum().item()) <= 1e-5 * (1 + (d * v).abs().sum().item())


# ------------------------------------------------------------------ all together
def step(ops, x, r, gain, w1, w2, offsets, targets):
    """A layer with experts and the loss, forward and backward, as in the graphs."""
    y, z = ops.layer_norm(x, gain, residual=r)
    h = torch.relu(ops.grouped_matmul(y, w1, offsets))
    logits = ops.grouped_matmul(h, w2, offsets) + z
    loss = ops.softmax_loss(logits, targets)
    (loss.sum() / len(targets)).backward()
    return loss


def test_autograd_matches_plain_gradients(ops):
    """The chain through torch.autograd against the same chain in fp32 torch operations."""
    g = gen(21)
    rows, width, inner = 96, 64, 80
    offsets = ranges([50, 0, 40], 2)
    targets = torch.randint(0, width, (rows,), generator=g, device="cuda")
    base = [rand(g, rows, width, dtype=HF), rand(g, rows, width, dtype=HF), rand(g, width, dtype=HF, scale=0.1, shift=1.0),
            rand(g, 3, inner, width, dtype=HF, scale=width ** -0.5), rand(g, 3, width, inner, dtype=HF, scale=inner ** -0.5)]
    mine = [t.clone().requires_grad_() for t in base]
    step(ops, *mine, offsets, targets)

    class Plain:
        @staticmethod
        def layer_norm(x, gain, residual):
            z = x + residual
            return torch.nn.functional.layer_norm(z, (width,), gain), z

        @staticmethod
        def grouped_matmul(x, w, offsets):
            y = [x.new_zeros(2, w.shape[1])]
            y += [x[a:b] @ w[e].t() for e, a, b in spans(offsets, rows)]
            y += [x.new_zeros(rows - int(offsets[-1]), w.shape[1])]
            return torch.cat(y)

        @staticmethod
        def softmax_loss(l, t):
            return torch.logsumexp(l, 1) - l.gather(1, t[:, None])[:, 0]

    plain = [t.float().requires_grad_() for t in base]
    step(Plain, *plain, offsets, targets)
    for m, p in zip(mine, plain):
        # every intermediate is rounded to half precision (2^-11): five roundings deep, each of the layer's scale
        assert (m.grad.float() - p.grad).norm() <= 16 * U[HF] * p.grad.norm() + 1e-6


def test_second_derivatives_are_refused(ops):
    x = torch.randn(4, 8, device="cuda", requires_grad=True)
    gain = torch.ones(8, device="cuda", requires_grad=True)
    for y in (ops.layer_norm(x, gain).square().sum(), ops.softmax_loss(x, torch.arange(4, device="cuda")).square().sum()):
        grad, = torch.autograd.grad(y, x, create_graph=True)
        with pytest.raises(RuntimeError):
            grad.sum().backward()


def test_another_stream_and_graph_replays(ops):
    """The same results on a side stream, and from every replay of a captured graph."""
    g = gen(22)
    x, r, gain = rand(g, 200, 512, dtype=BF), rand(g, 200, 512, dtype=BF), rand(g, 512, shift=1.0)
    w = rand(g, 5, 264, 512, dtype=BF, scale=0.05)
    offsets = ranges([40, 0, 90, 13, 50], 0)
    targets = torch.randint(0, 264, (200,), generator=g, device="cuda")
    dloss = torch.full((), 1 / 200, device="cuda")

    def run():
        y, z, mean, rstd = ops.layer_norm_forward(x, gain, residual=r)
        logits = ops.grouped_matmul_forward(y, w, offsets)
        loss, lse, d = ops.softmax_loss_grad(logits, targets, dloss)
        dy, dw = ops.grouped_matmul_backward(d, y, w, offsets, grad_dtype=SF)
        return [y, z, logits, loss, lse, d, dw, *ops.layer_norm_backward(dy, z, gain, mean, rstd)]

    want = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run()
    torch.cuda.synchronize()
    kept = x.clone()
    for turn in range(4):
        x.copy_(kept * (1 + turn))
        eager = [t.clone() for t in run()]
        for t in out:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), turn


def test_outputs_keep_to_their_rows(ops):
    """Through the C ABI with wider output rows: what lies between them is untouched."""
    L = ops.load()
    g = gen(23)
    rows, width, n = 70, 130, 140
    mark = 7.5
    x, gain = rand(g, rows, width, dtype=BF), rand(g, width, dtype=BF)
    stream = torch.cuda.current_stream().cuda_stream

    def room(rows, cols, dtype=BF):
        return torch.full((rows + 2, cols + 6), mark, dtype=dtype, device="cuda")

    def untouched(t, cols):
        return bool((t[0] == mark).all() and (t[-1] == mark).all() and (t[:, cols:] == mark).all())

    y, z, m = room(rows, width), room(rows, width), torch.empty(2, rows, device="cuda")
    ld = y.stride(0)
    assert L.pase_layer_norm_forward(0, 0, rows, width, x.data_ptr(), width, x.data_ptr(), width, gain.data_ptr(), None, 1e-5,
                                     y[1:].data_ptr(), ld, z[1:].data_ptr(), ld, m[0].data_ptr(), m[1].data_ptr(), stream) == 0
    ref = ops.layer_norm_forward(x, gain, residual=x)
    assert torch.equal(y[1:-1, :width], ref[0]) and torch.equal(z[1:-1, :width], ref[1])
    assert untouched(y, width) and untouched(z, width)
    w, offsets = rand(g, 2, n, width, dtype=BF), ranges([30, 33], 2)
    out = room(rows, n)
    assert L.pase_grouped_matmul_forward(0, 0, rows, 2, n, width, x.data_ptr(), width, w.data_ptr(), offsets.data_ptr(), 0,
                                         out[1:].data_ptr(), out.stride(0), stream) == 0
    assert torch.equal(out[1:-1, :n], ops.grouped_matmul_forward(x, w, offsets)) and untouched(out, n)
    dy, dx, dw = rand(g, rows, n, dtype=BF), room(rows, width), torch.full((2 * n * width + 64,), mark, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    assert L.pase_grouped_matmul_backward(0, 2, rows, 2, n, width, dy.data_ptr(), n, x.data_ptr(), width, w.data_ptr(),
                                          offsets.data_ptr(), 0, dx[1:].data_ptr(), dx.stride(0), dw.data_ptr(),
                                          ws.data_ptr(), ws.numel(), stream) == 0
    rx, rw = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=SF)
    assert torch.equal(dx[1:-1, :width], rx) and untouched(dx, width)
    assert torch.equal(dw[:-64].view(2, n, width), rw) and bool((dw[-64:] == mark).all())
    t, dloss = torch.randint(0, n, (rows,), generator=g, device="cuda"), torch.ones((), device="cuda")
    d, ll = room(rows, n), torch.empty(2, rows, device="cuda")
    assert L.pase_softmax_loss_grad(0, rows, n, out[1:].data_ptr(), out.stride(0), t.data_ptr(), 1, -100, dloss.data_ptr(), 0,
                                    ll[0].data_ptr(), ll[1].data_ptr(), d[1:].data_ptr(), d.stride(0), stream) == 0
    assert torch.equal(d[1:-1, :n], ops.softmax_loss_grad(out[1:-1, :n], t, dloss)[2]) and untouched(d, n)


def refused(ops, call):
    from paper_2407_04001_amd import PaseError
    with pytest.raises(PaseError) as e:
        call()
    return e.value.status == 1


def test_refused_tensors(ops):
    x = torch.zeros(4, 8, dtype=BF, device="cuda")
    gain, w = torch.ones(8, dtype=BF, device="cuda"), torch.zeros(2, 16, 8, dtype=BF, device="cuda")
    off, t = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    stat = torch.zeros(4, device="cuda")
    for call in (
            lambda: ops.layer_norm_forward(x.double(), gain), lambda: ops.layer_norm_forward(x[0], gain),
            lambda: ops.layer_norm_forward(x, gain[:7]), lambda: ops.layer_norm_forward(x, gain.half()),
            lambda: ops.layer_norm_forward(x, gain, gain.float()), lambda: ops.layer_norm_forward(x.t(), gain[:4]),
            lambda: ops.layer_norm_forward(x, gain, residual=x.float()), lambda: ops.layer_norm_forward(x, gain, residual=x[:3]),
            lambda: ops.layer_norm_forward(x, gain.cpu()), lambda: ops.layer_norm_forward(x[:1].expand(4, 8), gain),
            lambda: ops.layer_norm_backward(x, x, gain, stat.double(), stat), lambda: ops.layer_norm_backward(x, x, gain, stat[:3], stat),
            lambda: ops.grouped_matmul_forward(x.float(), w.float(), off), lambda: ops.grouped_matmul_forward(x, w.half(), off),
            lambda: ops.grouped_matmul_forward(x, w.transpose(1, 2), off), lambda: ops.grouped_matmul_forward(x[:, :7], w, off),
            lambda: ops.grouped_matmul_forward(x, w, off[:2]), lambda: ops.grouped_matmul_forward(x, w, off.float()),
            lambda: ops.grouped_matmul_forward(x, w, off.cpu()), lambda: ops.grouped_matmul_forward(x, w, off, out_dtype=HF),
            lambda: ops.grouped_matmul_backward(x, x, w, off), lambda: ops.grouped_matmul_forward(x, w[0], off),
            lambda: ops.softmax_loss_forward(x, t[:3]), lambda: ops.softmax_loss_forward(x, t.float()),
            lambda: ops.softmax_loss_grad(x, t, stat.double()), lambda: ops.softmax_loss_grad(x, t, stat[:2]),
            lambda: ops.softmax_loss_grad(x, t, stat, out=x.float()), lambda: ops.softmax_loss_backward(stat, x, t, stat[:2])):
        assert refused(ops, call)


@pytest.mark.parametrize("saved_by", ["softmax_loss", "tanh"])
@pytest.mark.parametrize("form", ["grad", "backward"])
def test_gradient_in_place_is_known_to_autograd(ops, form, saved_by):
    """A gradient written over logits that another node saved for its backward pass: that pass raises."""
    g = gen(31)
    base = rand(g, 6, 40).requires_grad_()
    targets = torch.randint(0, 40, (6,), generator=g, device="cuda")
    logits = torch.tanh(base)
    y = ops.softmax_loss(logits, targets).sum() if saved_by == "softmax_loss" else logits.sum()
    over, dloss = logits.detach(), torch.ones((), device="cuda")
    if form == "grad":
        ops.softmax_loss_grad(over, targets, dloss, out=over)
    else:
        ops.softmax_loss_backward(dloss, over, targets, ops.softmax_loss_forward(over, targets)[1], out=over)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_gradient_into_an_inference_tensor(ops):
    """These have no version to raise."""
    with torch.inference_mode():
        out = torch.empty(3, 10, device="cuda")
    logits, targets, dloss = torch.randn(3, 10, device="cuda"), torch.arange(3, device="cuda"), torch.ones((), device="cuda")
    assert torch.equal(ops.softmax_loss_grad(logits, targets, dloss, out=out)[2], ops.softmax_loss_grad(logits, targets, dloss)[2])


@pytest.mark.parametrize("dtype,param", [(BF, BF), (BF, SF), (SF, SF)])
@pytest.mark.parametrize("width", [5, 61, 342, 1022, 2050, 8193])
def test_norm_backward_where_mean_over_deviation_overflows(ops, width, dtype, param):
    """Constant rows of 2e36: their deviations are 0, mean * rstd is past fp32's range."""
    g = gen(width)
    z = torch.full((3, width), 2e36, dtype=dtype, device="cuda")
    mean = z[:, 0].float().contiguous()
    rstd = torch.full((3,), 1e-5 ** -0.5, device="cuda")
    dy, gain = rand(g, 3, width, dtype=dtype), rand(g, width, dtype=param, scale=0.3, shift=1.0)
    dx, dgain, dbias = ops.layer_norm_backward(dy, z, gain, mean, rstd)
    # h is 0, so that dx is rstd (dh - avg(dh)); the sum's and the products' roundings, as in the definition's bound
    dh = dy.double() * gain.double()
    r = rstd.double()[:, None]
    want = r * (dh - dh.mean(1, keepdim=True))
    tol = r * ((width + 8) * E * dh.abs().mean(1, keepdim=True) + 6 * E * (dh.abs() + dh.mean(1, keepdim=True).abs())) + 2 * E * want.abs()
    close(dx, want, tol, "dx")
    assert not dgain.any()
    close(dbias, dy.double().sum(0), 11 * E * dy.double().abs().sum(0), "dbias")


def loss_bounds(logits, targets, dloss):
    """loss64's loss and gradient, with bounds that do not grow with an offset that all logits of a row share.

    In fp32: x = l - max (off by e |x|); the sum of its exponentials (each off by 2 e (|x| + 4) of itself, and n e
    in the summing); the log of that; then exp(x - log sum), whose exponent is off by e |x| and e of itself again."""
    loss, _, d, _, _, _ = loss64(logits, targets, dloss)
    l = logits.double()
    x = l - l.max(1, keepdim=True).values
    p, logsum = torch.softmax(l, 1), torch.logsumexp(x, 1)
    far = -x.gather(1, targets[:, None])[:, 0]
    sum_err = (p * (x.abs() + 4) * 2 * E).sum(1) + (l.shape[1] + 8) * E + 2 * E * logsum
    loss_err = sum_err + 2 * E * (far + loss.abs())
    rel = 4 * E * (x.abs() + logsum[:, None] + 2) + sum_err[:, None]
    return loss, d, loss_err, p * rel * dloss.double().expand(len(l))[:, None].abs() + 4 * E * d.abs()


@pytest.mark.parametrize("shift", [0.0, 1e3, -1e6])
@pytest.mark.parametrize("rows,classes", [(9, 64), (9, 5000), (5, 40000), (600, 17000)])
def test_softmax_loss_of_shifted_logits(ops, rows, classes, shift):
    """An offset common to a row's logits changes neither its loss nor its gradient, also where the target is far
    above the rest and both are small."""
    g = gen(classes)
    logits = rand(g, rows, classes, scale=3.0)
    targets = torch.randint(0, classes, (rows,), generator=g, device="cuda")
    sure = torch.arange(0, rows, 2, device="cuda")
    logits[sure, targets[sure]] = logits[sure].max(1).values + 15
    logits += shift
    dloss = rand(g, rows)
    loss, d, el, ed = loss_bounds(logits, targets, dloss)
    close(ops.softmax_loss_forward(logits, targets)[0], loss, el, "loss")
    got, _, grad = ops.softmax_loss_grad(logits, targets, dloss)
    close(got, loss, el, "loss, with the gradient")
    close(grad, d, ed, "dlogits")
    over = logits.clone()
    ops.softmax_loss_grad(over, targets, dloss, out=over)
    assert torch.equal(over, grad)
    leaf = logits.clone().requires_grad_()
    ops.softmax_loss(leaf, targets).backward(dloss)
    close(leaf.grad, d, ed, "dlogits, autograd")


@pytest.mark.parametrize("classes", [600, 40000])
@pytest.mark.parametrize("dtype", [BF, HF, SF])
def test_lse_in_two_parts(ops, classes, dtype):
    """lse is as without its second part; the two together are the log-sum-exp to more than fp32; rows that are masked,
    ignored, out of range or NaN keep their rules in the gradient from both."""
    g = gen(classes + 1)
    logits, targets = rand(g, 9, classes, dtype=dtype, shift=500.0), torch.randint(0, classes, (9,), generator=g, device="cuda")
    logits[1] = -INF                              # no class left
    logits[2, classes // 2:] = -INF               # the target is masked
    targets[2] = classes - 1
    logits[3] = float("nan")                      # ignored
    targets[3], targets[4] = -100, classes        # ignored, out of range
    logits[5, 7] = float("nan")
    logits[6] = -INF
    logits[6, 3] = float("nan")                   # nothing but NaN and masked classes
    dloss = rand(g, 9)
    loss, lse, low = ops.softmax_loss_forward(logits, targets, low=True)
    plain = ops.softmax_loss_forward(logits, targets)
    assert torch.equal(loss.nan_to_num(1e9), plain[0].nan_to_num(1e9)) and torch.equal(lse.nan_to_num(1e9), plain[1].nan_to_num(1e9))
    keep = [0, 2, 4, 7, 8]
    x = logits.double()
    x = x - x.max(1, keepdim=True).values
    p = torch.softmax(x, 1).nan_to_num(0, 0, 0)
    logsum = torch.logsumexp(x, 1)
    err = (p * (x.abs().nan_to_num(0, 0, 0) + 4) * 2 * E).sum(1) + (classes + 8) * E + 2 * E * logsum
    off = (lse.double() + low.double() - torch.logsumexp(logits.double(), 1)).abs()
    assert (off[keep] <= err[keep]).all() and (low[keep].abs() <= E * lse[keep].abs() * 1.01).all()
    assert lse[1] == -INF and low[1] == 0 and loss[1] == INF and lse[3] == 0 and low[3] == 0 and loss[3] == 0
    one, _, d = ops.softmax_loss_grad(logits, targets, dloss)
    both = ops.softmax_loss_backward(dloss, logits, targets, lse, lse_low=low)
    assert torch.equal(one.nan_to_num(1e9), loss.nan_to_num(1e9))
    for t in (d, both):
        assert not t[1].any() and not t[3].any() and t[[4, 5, 6]].isnan().all() and torch.isfinite(t[[0, 2, 7, 8]]).all()
        assert abs(t[2, classes - 1] + dloss[2]) <= U[dtype] * dloss[2].abs()
    over = logits.clone()
    assert torch.equal(ops.softmax_loss_backward(dloss, over, targets, lse, out=over, lse_low=low).nan_to_num(1e9), both.nan_to_num(1e9))
    over = logits.clone()
    assert torch.equal(ops.softmax_loss_grad(over, targets, dloss, out=over)[2].nan_to_num(1e9), d.nan_to_num(1e9))


def test_arguments_by_name(ops):
    g = gen(33)
    x, gain, w = rand(g, 5, 8, dtype=BF), rand(g, 8, dtype=BF), rand(g, 2, 6, 8, dtype=BF)
    offsets, targets, dloss = ranges([2, 3]), torch.arange(5, device="cuda"), torch.ones((), device="cuda")
    y, z, mean, rstd = ops.layer_norm_forward(x, gain)
    dy = rand(g, 5, 6, dtype=BF)
    loss, lse = ops.softmax_loss_forward(x, targets)
    for a, b in (
            (ops.layer_norm_forward(gain=gain, x=x)[0], y),
            (ops.layer_norm_backward(dy=y, z=z, gain=gain, mean=mean, rstd=rstd)[0], ops.layer_norm_backward(y, z, gain, mean, rstd)[0]),
            (ops.grouped_matmul_forward(x=x, w=w, offsets=offsets), ops.grouped_matmul_forward(x, w, offsets)),
            (ops.grouped_matmul_backward(dy=dy, x=x, w=w, offsets=offsets)[1], ops.grouped_matmul_backward(dy, x, w, offsets)[1]),
            (ops.softmax_loss_forward(logits=x, targets=targets)[0], loss),
            (ops.softmax_loss_grad(targets=targets, logits=x, dloss=dloss)[2], ops.softmax_loss_grad(x, targets, dloss)[2]),
            (ops.softmax_loss_backward(dloss=dloss, logits=x, targets=targets, lse=lse), ops.softmax_loss_backward(dloss, x, targets, lse))):
        assert torch.equal(a, b)


def periodic(t, rows):
    """t's rows over and over, `rows` of them (a multiple of its own)."""
    return t.unsqueeze(0).expand(rows // len(t), *t.shape).reshape(rows, *t.shape[1:])


def repeats(big, small):
    """Whether big is small over and over."""
    return all(bool((part.view(-1, *small.shape) == small).all()) for part in big.split(len(small) << 12))


def test_norm_of_more_rows_than_one_launch_holds(ops):
    """2^29 rows of 8: 32 rows a workgroup of 256 are more than 2^32 - 1 threads."""
    g = gen(35)
    x, res, gain = rand(g, 4096, 8, dtype=BF), rand(g, 4096, 8, dtype=BF), rand(g, 8, dtype=BF, shift=1.0)
    few = ops.layer_norm_forward(x, gain, residual=res)
    rows = (1 << 29) + 4096
    many = ops.layer_norm_forward(periodic(x, rows), gain, residual=periodic(res, rows))
    for a, b in zip(many, few):
        assert a.shape[0] == rows and repeats(a, b)


@pytest.mark.parametrize("each", [True, False])
def test_softmax_loss_of_more_rows_than_one_launch_holds(ops, each):
    """2^26 rows of a wave each, and their gradients by workgroups of 256."""
    g = gen(36)
    logits, targets = rand(g, 4096, 24, dtype=BF, scale=2.0), torch.randint(0, 24, (4096,), generator=g, device="cuda").int()
    targets[5] = -100
    dloss = rand(g, 4096) if each else torch.full((), 0.5, device="cuda")
    loss, lse, low = ops.softmax_loss_forward(logits, targets, low=True)
    d, both = ops.softmax_loss_grad(logits, targets, dloss)[2], ops.softmax_loss_backward(dloss, logits, targets, lse, lse_low=low)
    rows = (1 << 26) + 4096
    logits, targets = periodic(logits, rows), periodic(targets, rows)
    dloss = periodic(dloss, rows) if each else dloss
    for a, b in zip(ops.softmax_loss_forward(logits, targets, low=True), (loss, lse, low)):
        assert repeats(a, b)
    assert repeats(ops.softmax_loss_backward(dloss, logits, targets, periodic(lse, rows), lse_low=periodic(low, rows)), both)
    assert all(repeats(a, b) for a, b in zip(ops.softmax_loss_grad(logits, targets, dloss, out=logits), (loss, lse, d)))


def test_product_of_more_tiles_than_one_launch_holds(ops):
    """512 groups of one row each and 2^20 columns: 17.9 million workgroups of 256."""
    g = gen(37)
    groups, n, k = 512, 1 << 20, 8
    x, w = whole(g, groups, k, dtype=BF), whole(g, 8, n, k, dtype=BF)
    offsets = torch.arange(groups + 1, dtype=torch.int32, device="cuda")
    y = ops.grouped_matmul_forward(x, periodic(w, groups), offsets)
    for t in range(groups):
        want = (w[t % 8].float() * x[t].float()).sum(1)      # whole numbers below 2^24: exact
        assert torch.equal(y[t], want.to(BF)), t


@pytest.mark.parametrize("pad", [0, 8, 3])
@pytest.mark.parametrize("rows,n,k", [(50, 24, 40), (3000, 520, 264), (3000, 1024, 1030)])
@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
def test_product_clamped_offsets(ops, rows, n, k, pad, dtype):
    """Offsets that leave 0 .. rows or fall below an earlier one are those of the nearest that keep the rule."""
    g = gen(rows + n)
    x, dy = wide(whole(g, rows, k, dtype=BF), pad), wide(whole(g, rows, n, dtype=BF), pad)
    w = whole(g, 4, n, k, dtype=BF)
    a, b = rows // 5, rows // 2
    for given, taken in (([-5, a, rows + 40, 7, b], [0, a, rows, rows, rows]), ([a, b, a - 3, b + 9, -1], [a, b, b, b + 9, b + 9]),
                         ([rows + 1, 0, 0, 0, 0], [rows] * 5), ([-9] * 5, [0] * 5), ([7, -2 ** 31, 2 ** 31 - 1, 0, 3], [7, 7, rows, rows, rows])):
        offsets, as_if = (torch.tensor(o, dtype=dtype, device="cuda") for o in (given, taken))
        y, _ = product64(x, w, as_if)
        assert torch.equal(ops.grouped_matmul_forward(x, w, offsets, out_dtype=SF), y.float())
        dx, dw, _, _ = product_grad64(dy, x, w, as_if)
        gx, gw = ops.grouped_matmul_backward(dy, x, w, offsets, grad_dtype=SF)
        assert torch.equal(gx, dx.to(BF)) and torch.equal(gw, dw.float())


def test_norm_constant_row_whose_squares_overflow(ops):
    """y of a constant row is the bias, whatever fp32 makes of the square of its mean's rounding."""
    x = torch.full((2, 300), 1e30, device="cuda")
    gain, bias = torch.rand(300, device="cuda") + 0.5, torch.randn(300, device="cuda")
    y, _, mean, rstd = ops.layer_norm_forward(x, gain, bias, eps=1e-5)
    tol = 308 * E * 1e30
    close(mean, x[:, 0].double(), tol, "mean")
    assert torch.equal(y, bias.expand(2, 300))


def test_one_row_of_a_wide_buffer(ops):
    """The distance between rows does not matter where there is one."""
    g = gen(34)
    buffer = torch.zeros(2, 5_000_000, dtype=BF, device="cuda")
    x = buffer[1:, :64]
    x.copy_(rand(g, 1, 64))
    w, offsets = rand(g, 1, 16, 64, dtype=BF), ranges([1])
    dy = rand(g, 1, 16, dtype=BF)
    assert torch.equal(ops.grouped_matmul_forward(x, w, offsets), ops.grouped_matmul_forward(x.clone(), w, offsets))
    for a, b in zip(ops.grouped_matmul_backward(dy, x, w, offsets), ops.grouped_matmul_backward(dy, x.clone(), w, offsets)):
        assert torch.equal(a, b)
