"""The operators that run on a tile between two redistributions: linear layer, layer norm (both with their
gradients) and orthogonalisation.

Results are compared with the definition in 64 bits.  Tolerances are derived, element by element where the
operator is a sum: an output rounded once to a type with p significant bits is off by 2^-p of itself; a sum of
k products accumulated in 32 bits by at most k 2^-23 of the sum of the products' magnitudes (a product of two
16-bit floats is exact in 32 bits; each addition, rounded or truncated, loses at most 2^-23 of a partial sum);
and what passes through an activation by that times its steepest slope.
"""
import ctypes
import math

import pytest

from paper_2112_01075_b200 import api

torch = pytest.importorskip("torch")

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_ULP = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}      # 2^-p of a value, rounding to nearest
TINY = {BF16: 2.0 ** -134, F16: 2.0 ** -25, F32: 2.0 ** -150}       # ... of a subnormal
STEEPEST = {"none": 1.0, "relu": 1.0, "gelu": 1.13, "silu": 1.1}


@pytest.fixture(autouse=True)
def no_wait_runs_out(request):
    """No test may leave a bounded wait behind that ran out (but the one that makes them)."""
    counts = "gpu" in request.keywords and "runs_out" not in request.node.name
    before = api.redist_product_timeouts() if counts else 0
    yield
    assert not counts or api.redist_product_timeouts() == before


def rand(g, *shape, scale=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def act64(z, name):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def within(got, want, slack, dtype):
    """|got - want| <= rounding to dtype + slack, element by element; NaN where NaN is wanted."""
    bound = want.abs() * HALF_ULP[dtype] * 1.001 + slack * 1.01 + TINY[dtype]
    off = (got.double() - want).abs()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    bad = (off > bound) & ~torch.isnan(want) & ~(got.double() == want)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((off / bound)[bad].max()):.2f} of the bound"


def products(a, b):
    """a b^T in 64 bits and the error bound of its accumulation in 32."""
    a, b = a.double(), b.double()
    return a @ b.T, (a.shape[1] + 2) * 2.0 ** -23 * (a.abs() @ b.abs().T)


# ---- linear -----------------------------------------------------------------------------------------------

LINEAR = [  # rows, in, out
    (1, 1, 1), (1, 64, 256), (2, 7, 3), (3, 4096, 130), (5, 4104, 777), (8, 1000, 96), (9, 128, 4096), (16, 512, 640),
    (17, 8200, 264), (33, 72, 2000), (64, 1024, 1024), (65, 65, 65), (127, 129, 255), (128, 64, 256), (129, 200, 300),
    (256, 256, 256), (300, 1021, 515), (777, 96, 1030), (1000, 333, 2047), (2048, 512, 768), (4099, 80, 24),
]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,n", LINEAR)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_linear_forward(rows, k, n, dtype):
    g = gen(rows * 7 + k * 3 + n)
    x, w = rand(g, rows, k, dtype=dtype), rand(g, n, k, scale=k ** -0.5, dtype=dtype)
    which = (rows + k + n) % 4
    activation = api.ACTIVATIONS[which]
    bias = rand(g, n, dtype=(BF16, F16, F32)[(rows + n) % 3])
    residual = rand(g, rows, n, dtype=dtype)
    z, slack = products(x, w)
    within(api.linear_forward(x, w), z, slack, dtype)
    pre = torch.full((rows, n), float("nan"), dtype=dtype, device="cuda")
    y = api.linear_forward(x, w, bias, residual, activation, pre=pre)
    z = z + bias.double()
    slack = slack + 2.0 ** -23 * z.abs()
    within(pre, z, slack, dtype)
    want = act64(z, activation) + residual.double()
    slack = slack * STEEPEST[activation] + 2.0 ** -20 * (z.abs() + want.abs())     # erf and exp: a few units of 32 bits
    within(y, want, slack, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("activation", api.ACTIVATIONS)
def test_activations_over_their_whole_range(activation):
    """One column, weight 1: the activation of every bf16 number of up to 2^7, of infinities and of NaN."""
    z = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(BF16).cuda()
    z = z[(z.abs() <= 128) | ~torch.isfinite(z)].reshape(-1, 1).contiguous()
    one = torch.ones((1, 1), dtype=BF16, device="cuda")
    y = api.linear_forward(z, one, activation=activation)
    z64 = z.double()
    want = act64(z64, activation)
    if activation in ("gelu", "silu"):
        want = torch.where(z64 == -math.inf, y.double(), want)         # -inf * 0: NaN by the product, 0 by the limit
    # what comes out of 1 + erf or out of the quotient is off by a few units of 32 bits of z
    within(y, want, z64.abs().nan_to_num(0, 0, 0) * 2.0 ** -21, BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_gelu_keeps_its_relative_accuracy_below_zero(dtype):
    """Every number of the type between -14 and 14, forward and slope.  Computed in 32 bits: Phi(z) for z < 0 is exp(-z^2 / 2)
    times a factor of size 1 / |z|; that factor, the reciprocal in it and the power of two are off by a few 2^-23, together by
    at most 2^-20 of the value, and the exponent, the rounded product of z, z and a constant, by 3 2^-24 of itself, z^2 / 2:
    1.5 z^2 2^-24 of the value.  32-bit results below 2^-126 may be flushed to zero."""
    z = torch.arange(0, 1 << 16, dtype=torch.int32).to(torch.int16).view(dtype).cuda()
    z = z[z.abs() <= 14].reshape(-1, 1).contiguous()
    one, z64 = torch.ones((1, 1), dtype=dtype, device="cuda"), z.double()
    of_itself = 2.0 ** -20 + 1.5 * z64 ** 2 * 2.0 ** -24
    phi = torch.exp(torch.special.log_ndtr(z64))
    want = z64 * phi
    within(api.linear_forward(z, one, activation="gelu"), want, want.abs() * of_itself + 2.0 ** -126, dtype)
    few = api.linear_forward(one, z, activation="gelu")                     # one row: the other kernel
    within(few.T, want, want.abs() * of_itself + 2.0 ** -126, dtype)
    slope, second = slope64(z64, "gelu"), z64 * torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    _, _, db = api.linear_backward(one.expand(1, z.shape[0]).contiguous(), one, z, z.T.contiguous(), "gelu", need=(False, False, True))
    within(db, slope[:, 0], ((phi + second.abs()) * of_itself)[:, 0] + 2.0 ** -126, F32)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,n", [(40, 96, 72), (300, 136, 520), (1, 256, 64), (6, 520, 90)])
def test_linear_strides_and_orders(rows, k, n):
    """Column-major operands, padded rows, bases off 16 bytes, outputs and residuals inside wider matrices."""
    g = gen(5)
    x0, w0 = rand(g, rows, k, dtype=BF16), rand(g, n, k, scale=0.1, dtype=BF16)
    r0 = rand(g, rows, n, dtype=BF16)
    z, slack = products(x0, w0)
    want = z + r0.double()

    def padded(t, extra, shift):
        big = torch.full((t.shape[0], t.shape[1] + extra + shift), float("nan"), dtype=t.dtype, device="cuda")
        view = big[:, shift:shift + t.shape[1]]
        view.copy_(t)
        return view

    orders = [lambda t: t, lambda t: t.T.contiguous().T, lambda t: padded(t, 8, 8), lambda t: padded(t, 5, 1),
              lambda t: padded(t.T.contiguous(), 3, 2).T]
    for ox in orders:
        for ow in orders:
            x, w = ox(x0), ow(w0)
            within(api.linear_forward(x, w, residual=r0), want, slack + 2.0 ** -23 * want.abs(), BF16)
    for shift, extra in ((8, 8), (1, 2), (0, 1)):
        big = torch.full((rows, n + extra + shift), 7.0, dtype=BF16, device="cuda")
        out = big[:, shift:shift + n]
        api.linear_forward(x0, w0, residual=padded(r0, 3, 1), out=out)
        within(out, want, slack + 2.0 ** -23 * want.abs(), BF16)
        assert bool((big[:, :shift] == 7).all()) and bool((big[:, shift + n:] == 7).all())
    inplace = r0.clone()
    assert api.linear_forward(x0, w0, residual=inplace, out=inplace) is inplace
    within(inplace, want, slack + 2.0 ** -23 * want.abs(), BF16)
    # two column blocks of one matrix: residual on the left, result on the right
    both = torch.zeros((rows, 2 * n), dtype=BF16, device="cuda")
    both[:, :n] = r0
    api.linear_forward(x0, w0, residual=both[:, :n], out=both[:, n:])
    within(both[:, n:], want, slack + 2.0 ** -23 * want.abs(), BF16)
    assert torch.equal(both[:, :n], r0)


@pytest.mark.gpu
def test_linear_not_a_number_stays_in_its_row_and_column():
    g = gen(8)
    for rows in (3, 200):
        x, w = rand(g, rows, 136, dtype=F16), rand(g, 300, 136, scale=0.1, dtype=F16)
        x[1, 5] = float("nan")
        x[2, 0] = float("inf")
        w[7, 3] = float("nan")
        y = api.linear_forward(x, w)
        clean = torch.ones(rows, 300, dtype=torch.bool, device="cuda")
        clean[1], clean[2], clean[:, 7] = False, False, False
        assert bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[:, 7]).all()) and not bool(torch.isfinite(y[2]).any())
        assert bool(torch.isfinite(y[clean]).all())
    assert float(api.linear_forward(torch.full((1, 1), float("nan"), dtype=F16, device="cuda"),
                                    torch.ones((1, 1), dtype=F16, device="cuda"), activation="relu")) != 0


GRAD = [(1, 1, 1), (1, 300, 70), (7, 64, 33), (64, 200, 128), (65, 65, 65), (200, 770, 301), (333, 128, 1001), (520, 96, 264),
        (1024, 512, 256), (2500, 40, 56)]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,n", GRAD)
@pytest.mark.parametrize("activation", api.ACTIVATIONS)
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_linear_backward(rows, k, n, activation, dtype):
    g = gen(rows + k + n)
    x, w = rand(g, rows, k, dtype=dtype), rand(g, n, k, scale=k ** -0.5, dtype=dtype)
    pre, dy = rand(g, rows, n, dtype=dtype), rand(g, rows, n, dtype=dtype)
    dx, dw, db = api.linear_backward(dy, x, w, pre if activation != "none" else None, activation)
    dz = dy.double() * slope64(pre.double(), activation)
    # dz is rounded to dtype before it is multiplied; the slope is off by a few units of 32 bits
    off = dz.abs() * HALF_ULP[dtype] * (activation != "none") + dy.double().abs() * 2.0 ** -20 + TINY[dtype]
    wa, xa = w.double().abs(), x.double().abs()
    within(dx, dz @ w.double(), off @ wa + (n + 2) * 2.0 ** -23 * (dz.abs() @ wa), dtype)
    within(dw, dz.T @ x.double(), off.T @ xa + (rows + 2) * 2.0 ** -23 * (dz.abs().T @ xa), dtype)
    within(db, dz.sum(0), (dy.double().abs() * 2.0 ** -20).sum(0) + (rows + 2) * 2.0 ** -24 * dz.abs().sum(0), F32)
    again = api.linear_backward(dy, x, w, pre, activation)
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))       # no order that changes from call to call


@pytest.mark.gpu
def test_linear_backward_parts_strides_and_no_rows():
    g = gen(3)
    rows, k, n = 90, 72, 104
    x, w, pre, dy = rand(g, rows, k, dtype=BF16), rand(g, n, k, dtype=BF16), rand(g, rows, n, dtype=BF16), rand(g, rows, n, dtype=BF16)
    full = api.linear_backward(dy, x, w, pre, "gelu")
    for need in ((True, False, False), (False, True, False), (False, False, True), (True, False, True)):
        part = api.linear_backward(dy, x, w, pre, "gelu", need=need)
        assert all((p is None) == (not want) and (p is None or torch.equal(p, f)) for p, want, f in zip(part, need, full))
    wide = torch.zeros((rows, 3 * n + 1), dtype=BF16, device="cuda")
    wide[:, 1:1 + n], wide[:, 2 * n:3 * n] = dy, pre
    got = api.linear_backward(wide[:, 1:1 + n], x.T.contiguous().T, w.T.contiguous().T, wide[:, 2 * n:3 * n], "gelu")
    assert all(torch.equal(a, b) for a, b in zip(got, full))
    got = api.linear_backward(wide[:, 1:1 + n], x, w)
    want = api.linear_backward(dy, x, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    none = torch.empty((0, n), dtype=BF16, device="cuda")
    dx, dw, db = api.linear_backward(none, torch.empty((0, k), dtype=BF16, device="cuda"), w, none, "silu")
    assert dx.shape == (0, k) and not bool(dw.any()) and not bool(db.any())
    assert api.linear_forward(torch.empty((0, k), dtype=BF16, device="cuda"), w).shape == (0, n)


@pytest.mark.gpu
@pytest.mark.parametrize("activation", api.ACTIVATIONS)
def test_linear_gradient_against_differences(activation):
    """L = <y, dy>; (L(x + hv) - L(x - hv)) / 2h against <dx, v>, and the same for w.  Inputs are multiples of 2^-6, so
    x +- hv is exact.  Central differences are off by h^2/6 of the third derivative along v; the outputs' rounding
    moves L by at most sum |y dy| 2^-11, which is divided by h."""
    g = gen(21)
    rows, k, n, h = 24, 16, 40, 2.0 ** -5
    grid = lambda *s: (torch.randint(-64, 65, s, generator=g, device="cuda") / 64)        # noqa: E731
    x, w, dy = grid(rows, k).to(F16), (grid(n, k) / 4).to(F16), grid(rows, n).to(F16)
    if activation == "relu":                                                             # no kink within reach
        z, xa, wa = x.double() @ w.double().T, x.double().abs().sum(1), w.double().abs().sum(1)
        dy = torch.where(z.abs() < 1.01 * h * torch.maximum(xa[:, None], wa[None]), torch.zeros_like(dy), dy)
        assert bool(dy.any())
    pre = torch.empty((rows, n), dtype=F16, device="cuda")
    y = api.linear_forward(x, w, activation=activation, pre=pre)
    dx, dw, _ = api.linear_backward(dy, x, w, pre, activation)
    for name in ("x", "w"):
        v = torch.randint(0, 2, (x if name == "x" else w).shape, generator=g, device="cuda").to(F16) * 2 - 1
        at = lambda s: (api.linear_forward(x + s * h * v, w, activation=activation) if name == "x"      # noqa: E731
                        else api.linear_forward(x, w + s * h * v, activation=activation)).double()
        got = float(((at(1) - at(-1)) * dy.double()).sum() / (2 * h))
        want = float(((dx if name == "x" else dw).double() * v.double()).sum())
        dzdv = (v.double() @ w.double().T if name == "x" else x.double() @ v.double().T).abs()
        slack = float((y.double() * dy.double()).abs().sum()) * 2.0 ** -11 / h * 1.1
        slack += float((dy.double().abs() * dzdv ** 3).sum()) * h * h / 6 * (1.2 if activation in ("gelu", "silu") else 0)
        # dx and dw are rounded, their operand dz is, and so is the z at which the slope is taken
        slack += 4 * 2.0 ** -11 * float((dy.double().abs() * dzdv).sum()) + 2.0 ** -11 * float((dx if name == "x" else dw).double().abs().sum())
        assert abs(got - want) <= slack, (name, got, want, slack)
        assert slack < 0.25 * float((dy.double().abs() * dzdv).sum())                    # the bound says something


# ---- layer norm ---------------------------------------------------------------------------------------------

NORM = [(1, 1), (3, 1), (1, 7), (5, 64), (9, 100), (130, 255), (64, 256), (33, 257), (17, 511), (300, 512), (1000, 1000),
        (77, 1024), (50, 1531), (40, 2048), (500, 4096), (11, 4100), (23, 8192), (7, 9001), (6, 16384), (5, 20011), (3, 40000),
        (2, 70001), (3000, 48)]


def norm_inputs(rows, cols, dtype, seed, mean=3.0):
    g = gen(seed)
    x = (rand(g, rows, cols) * torch.exp(rand(g, cols, scale=0.5)) + mean * rand(g, rows, 1)).to(dtype)
    return x, 1 + 0.1 * rand(g, cols), 0.1 * rand(g, cols), rand(g, rows, cols).to(dtype)


def norm64(x, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return mean, rstd, (x - mean[:, None]) * rstd[:, None]


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", NORM)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_layer_norm_forward(rows, cols, dtype):
    x, gamma, beta, _ = norm_inputs(rows, cols, dtype, rows * 31 + cols)
    wt = (BF16, F16, F32)[(rows + cols) % 3]
    gamma, beta = gamma.to(wt), beta.to(wt)
    y, mean, rstd = api.layer_norm_forward(x, gamma, beta, eps=1e-5)
    m64, r64, xh = norm64(x, 1e-5)
    # a sum of `cols` numbers, in chains of at most cols/32 + 64 additions; the mean's error moves every difference
    chain = (cols / 32 + 64) * 2.0 ** -24
    off_mean = x.double().abs().mean(1) * chain + m64.abs() * 2.0 ** -24
    within(mean, m64, off_mean, F32)
    off_rstd = r64 * (chain + 2.0 ** -22) + r64 * (off_mean * r64) ** 2 + r64 * 2 * off_mean * r64 * 2.0 ** -23
    within(rstd, r64, off_rstd, F32)
    slack = (xh.abs() * (off_rstd / r64)[:, None] + (off_mean * r64)[:, None] + (x.double().abs() * r64[:, None]) * 2.0 ** -24) * gamma.double().abs()
    want = xh * gamma.double() + beta.double()
    within(y, want, slack + 2.0 ** -22 * (want.abs() + beta.double().abs()), dtype)
    plain, _, _ = api.layer_norm_forward(x)
    within(plain, xh, slack / gamma.double().abs() + 2.0 ** -22 * xh.abs(), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", NORM)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_layer_norm_backward(rows, cols, dtype):
    x, gamma, _, dy = norm_inputs(rows, cols, dtype, rows * 17 + cols, mean=0.5)
    m64, r64, _ = norm64(x, 1e-5)
    mean, rstd = m64.float(), r64.float()
    dx, dg, db = api.layer_norm_backward(dy, x, gamma, mean, rstd)
    m, r = mean.double()[:, None], rstd.double()[:, None]
    xh, d = (x.double() - m) * r, dy.double()
    off_xh = 2.0 ** -23 * (xh.abs() + r * (x.double().abs() + m.abs()))
    c = d * gamma.double()
    s1, s2 = c.mean(1, keepdim=True), (c * xh).mean(1, keepdim=True)
    chain = (cols / 32 + 64) * 2.0 ** -24
    off1 = c.abs().mean(1, keepdim=True) * chain
    off2 = (c * xh).abs().mean(1, keepdim=True) * chain + (c.abs() * off_xh).mean(1, keepdim=True)
    want = (c - s1 - xh * s2) * r
    slack = r * (off1 + xh.abs() * off2 + off_xh * s2.abs() + 2.0 ** -22 * (c.abs() + s1.abs() + (xh * s2).abs()))
    within(dx, want, slack, dtype)
    chain = (rows + 16) * 2.0 ** -24
    within(dg, (d * xh).sum(0), (d * xh).abs().sum(0) * chain + (d.abs() * off_xh).sum(0), F32)
    within(db, d.sum(0), d.abs().sum(0) * chain, F32)
    again = api.layer_norm_backward(dy, x, gamma, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip((dx, dg, db), again))


@pytest.mark.gpu
def test_layer_norm_strides_means_and_special_values():
    g = gen(4)
    for dtype in (BF16, F32):
        for shift, extra in ((0, 3), (1, 0), (8, 8)):
            big = rand(g, 37, 300 + shift + extra, dtype=dtype)
            x = big[:, shift:shift + 300]
            wide = torch.full((37, 310 + shift), 7.0, dtype=dtype, device="cuda")
            out = wide[:, shift:shift + 300]
            y, mean, rstd = api.layer_norm_forward(x, out=out)
            # another split of the sums, the same formula: 1e-5 in 32 bits, and one unit of bf16 where that turns a rounding
            tol = 1e-5 if dtype == F32 else 2.0 ** -7
            assert torch.allclose(y.float(), api.layer_norm_forward(x.contiguous())[0].float(), atol=1e-5, rtol=tol)
            assert bool((wide[:, :shift] == 7).all()) and bool((wide[:, shift + 300:] == 7).all())
            dx, dg, db = api.layer_norm_backward(x, x, None, mean, rstd)
            dx2, dg2, db2 = api.layer_norm_backward(x.contiguous(), x.contiguous(), None, mean, rstd)
            assert torch.allclose(dx.float(), dx2.float(), atol=1e-5, rtol=tol)
            assert torch.allclose(dg, dg2, rtol=1e-5, atol=1e-4) and torch.allclose(db, db2, rtol=1e-5, atol=1e-4)
    # a mean far larger than the spread: no cancellation in the variance (1e4 + k/8 is exact in 32 bits)
    x = 1e4 + torch.randint(-8, 9, (20, 777), generator=g, device="cuda").float() / 8
    _, mean, rstd = api.layer_norm_forward(x)
    _, r64, _ = norm64(x, 1e-5)
    assert float(((rstd.double() - r64) / r64).abs().max()) < 2e-6
    # constant rows: the variance is zero
    y, mean, rstd = api.layer_norm_forward(torch.full((3, 500), 2.0, device="cuda"), eps=1e-5)
    assert not bool(y.any()) and bool((mean == 2).all()) and torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))
    # NaN and infinities stay in their rows
    x = rand(g, 9, 130, dtype=BF16)
    x[3, 4], x[5, 129] = float("nan"), float("inf")
    y, mean, rstd = api.layer_norm_forward(x)
    good = torch.tensor([i not in (3, 5) for i in range(9)], device="cuda")
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[5]).all()) and bool(torch.isfinite(y[good]).all())
    # no rows
    y, mean, rstd = api.layer_norm_forward(torch.empty((0, 8), device="cuda"))
    dx, dg, db = api.layer_norm_backward(y, y, None, mean, rstd)
    assert y.shape == (0, 8) and mean.shape == (0,) and not bool(dg.any()) and not bool(db.any())


@pytest.mark.gpu
def test_layer_norm_gradient_against_differences():
    """32-bit inputs: (L(x + hv) - L(x - hv)) / 2h against <dx, v>, likewise gamma and beta.  h = 2^-6; the central
    difference is off by about h^2 (1.6 % of 1.6 %), the outputs' rounding by |y dy| 2^-24 / h."""
    g = gen(12)
    rows, cols, h = 13, 200, 2.0 ** -6
    x, gamma, beta, dy = rand(g, rows, cols), 1 + 0.1 * rand(g, cols), rand(g, cols), rand(g, rows, cols)
    _, mean, rstd = api.layer_norm_forward(x, gamma, beta)
    dx, dg, db = api.layer_norm_backward(dy, x, gamma, mean, rstd)
    for what, grad in (("x", dx), ("gamma", dg), ("beta", db)):
        v = torch.randint(0, 2, grad.shape, generator=g, device="cuda").float() * 2 - 1
        args = {"x": x, "gamma": gamma, "beta": beta}
        at = lambda s: api.layer_norm_forward(**{k: t + s * h * v if k == what else t for k, t in args.items()})[0].double()   # noqa: E731
        got = float(((at(1) - at(-1)) * dy.double()).sum() / (2 * h))
        want = float((grad.double() * v.double()).sum())
        scale = float(dy.double().abs().sum())
        assert abs(got - want) <= scale * (4 * h * h + 4 * 2.0 ** -24 / h), (what, got, want)


# ---- orthogonalisation ------------------------------------------------------------------------------------------

MUON = (3.4445, -4.7750, 2.0315)


def orthogonalize64(x, steps=5, coefficients=MUON, eps=1e-7, scale=1.0):
    x = x.double()
    if x.dim() == 2:
        return orthogonalize64(x[None], steps, coefficients, eps, scale)[0]
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + eps)
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    for k in range(steps):
        a, b, c = coefficients[k] if hasattr(coefficients[0], "__len__") else coefficients
        gram = x @ x.mT
        x = a * x + (b * gram + c * gram @ gram) @ x
    return scale * (x.mT if tall else x)


def gradient_like(g, batch, m, n, kind):
    if kind == "gaussian":
        return rand(g, batch, m, n)
    r = max(1, min(m, n) // 16)
    if kind == "one direction":
        return rand(g, batch, m, 1) @ rand(g, batch, 1, n) + 0.003 * rand(g, batch, m, n)
    return (rand(g, batch, m, r) * torch.logspace(0, -1.5, r, device="cuda")) @ rand(g, batch, r, n) + 0.1 * rand(g, batch, m, n)


# The output's rounding to bf16 is 2^-9 / sqrt(3) = 1.1e-3 of a value in the worst place of a binade, 1.7e-3 of the
# norm on average over one; f16 operands add 2^-12 of each of a step's three operands, which the last two or three
# steps, where the slope of the polynomial is about 1 to 3, pass on: about 2^-12 (1 + 3 + 9) / sqrt(3) = 1.8e-3.
# Together sqrt(1.7^2 + 1.8^2) = 2.5e-3; twice that is allowed.
ORTHOGONAL = 5e-3
# That averages over many elements.  A handful has the worst case: per step at most 2^-11 (2 |B| + |b| + 2 |c|) = 7e-3 of
# the value, passed on by the four later steps with slopes of up to 1.4 on the cycle 0.7 ... 1.12 of a singular value:
# 7e-3 (1 + 1.3 + 1.4 + 1.9 + 2.2) + 2^-8.
ORTHOGONAL_FEW = 6e-2


@pytest.mark.gpu
@pytest.mark.parametrize("batch,m,n", [(1, 1, 1), (3, 1, 40), (2, 40, 1), (1, 8, 8), (2, 33, 65), (5, 64, 64), (1, 100, 300),
                                       (1, 300, 100), (2, 128, 128), (3, 129, 257), (1, 520, 1111), (1, 1111, 520), (2, 512, 512),
                                       (1, 640, 2056), (9, 96, 80)])
@pytest.mark.parametrize("kind", ["gaussian", "low rank", "one direction"])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_orthogonalize(batch, m, n, kind, dtype):
    x = (gradient_like(gen(m + n), batch, m, n, kind) * 2.0 ** -7).to(dtype)
    got, want = api.orthogonalize(x), orthogonalize64(x)
    assert got.dtype == BF16 and got.shape == x.shape
    for i in range(batch):
        off = float((got[i].double() - want[i]).norm() / want[i].norm())
        assert off < (ORTHOGONAL if min(m, n) >= 8 else ORTHOGONAL_FEW), off
    assert torch.equal(got, api.orthogonalize(x))
    assert torch.equal(got[0], api.orthogonalize(x[0]))


# Part of the directions strong and equal, the rest noise.  f16 rounds the operands to 2e-4 of themselves (2^-10 / sqrt(12) over
# the mean of a binade); A's error passes into X with |b + 2 c A| = 1.2, B's and X's with |B| = 2.8: 8e-4 of the norm a step
# where the strong directions have settled, passed on by each later step with the polynomial's slope there, about 1.4, all of them
# alike here: 8e-4 sqrt(1 + 2 + 4 + 8) = 3.2e-3; with the output's 1.7e-3 3.6e-3.  A tenth more is allowed.
ORTHOGONAL_PARTIAL = 4e-3


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(64, 128), (128, 128), (128, 256), (256, 128), (256, 256), (512, 512)])
@pytest.mark.parametrize("part", [0.25, 0.5, 0.75])
@pytest.mark.parametrize("noise", [1e-2, 1e-3])
def test_orthogonalize_part_of_the_directions_strong(m, n, part, noise):
    g = gen(m + n)
    small, rank = min(m, n), round(part * min(m, n))
    u, _ = torch.linalg.qr(rand(g, 2, m, small))
    v, _ = torch.linalg.qr(rand(g, 2, n, small))
    x = (u[..., :rank] @ v[..., :rank].mT + noise * max(m, n) ** -0.5 * rand(g, 2, m, n)).to(BF16)
    got, want = api.orthogonalize(x), orthogonalize64(x)
    for i in range(2):
        off = float((got[i].double() - want[i]).norm() / want[i].norm())
        assert off < ORTHOGONAL_PARTIAL, off


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(8, 1 << 20), (3 << 18, 16)])
def test_orthogonalize_long_rows(m, n):
    """The tensor cores add 16 products at a time and cut each sum off to 24 bits: at most 2^-23 of a sum that is half of the
    last on average, so A is small by up to k 2^-28; b A + 2 c A A, about 1.4 of that, goes into X, and the steps pass it on."""
    x = rand(gen(n), m, n, dtype=BF16)
    got, want = api.orthogonalize(x), orthogonalize64(x)
    off = float((got.double() - want).norm() / want.norm())
    assert off < ORTHOGONAL + 2 * max(m, n) * 2.0 ** -28, off


@pytest.mark.parametrize("rows,cols", [(1, (1 << 31) - 600), ((1 << 31) - 600, 1), (1, (1 << 22) + 1), ((1 << 22) + 1, 8)])
def test_orthogonalize_refuses_sums_that_32_bits_do_not_hold(rows, cols):
    abc = (ctypes.c_float * 3)(*MUON)
    op = api._Orthogonal(1, rows, cols, 0, 1, 1e-7, 1.0, 0, (0x10000, cols, 1), (0x900000000, cols, 1), 0, 0, ctypes.addressof(abc))
    assert api.load().redist_orthogonalize(op, None, 0, None) == 10 and api.load().redist_orthogonalize_scratch_bytes(op) == 0


@pytest.mark.gpu
def test_orthogonalize_options_and_strides():
    g = gen(6)
    x = rand(g, 3, 70, 90, dtype=BF16)
    per_step = [(4.0, -6.0, 3.0), (3.0, -3.2, 1.2), (1.5, -0.5, 0.0)]
    for kw in (dict(steps=1), dict(steps=3), dict(steps=12), dict(scale=0.2), dict(eps=1.0), dict(steps=3, coefficients=per_step),
               dict(steps=15, coefficients=(1.5, -0.5, 0.0))):
        got, want = api.orthogonalize(x, **kw), orthogonalize64(x, **kw)
        assert float((got.double() - want).norm() / want.norm()) < ORTHOGONAL * (2 if kw.get("steps", 5) > 5 else 1), kw
    # after enough cubic steps the rows are orthonormal
    q = api.orthogonalize(x, steps=25, coefficients=(1.5, -0.5, 0.0)).double()
    assert float((q @ q.mT - torch.eye(70, device="cuda", dtype=torch.float64)).norm() / math.sqrt(3 * 70)) < 2e-2
    wide = torch.full((3, 80, 101), 7.0, dtype=BF16, device="cuda")
    wide[:, 2:72, 1:91] = x
    out = torch.full((3, 71, 95), 7.0, dtype=BF16, device="cuda")
    api.orthogonalize(wide[:, 2:72, 1:91], out=out[:, :70, 3:93])
    assert torch.equal(out[:, :70, 3:93], api.orthogonalize(x))
    assert bool((out[:, 70] == 7).all()) and bool((out[..., :3] == 7).all()) and bool((out[..., 93:] == 7).all())
    assert api.orthogonalize(torch.empty((0, 4, 4), device="cuda")).shape == (0, 4, 4)


@pytest.mark.gpu
def test_orthogonalize_scale_of_the_input_and_special_values():
    g = gen(7)
    x = rand(g, 4, 48, 80)
    want = api.orthogonalize(x)
    for power in (-60, -40, 60, 110):                   # norms from 5e-17, where eps still does not count, to 8e34
        y = x * 2.0 ** power
        got, exact = api.orthogonalize(y, eps=1e-30), orthogonalize64(x, eps=0.0)
        assert float((got.double() - exact).norm() / exact.norm()) < ORTHOGONAL
    x[1] = 0
    x[2, 3, 4] = float("nan")
    x[3, 0, 0] = float("inf")
    got = api.orthogonalize(x)
    assert torch.equal(got[0], want[0]) and not bool(got[1].any())
    assert bool(torch.isnan(got[2]).all()) and bool(torch.isnan(got[3]).all())


# ---- offsets beyond 32 bits -------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("stride", [(1 << 26) + 8, (1 << 26) + 1])
def test_rows_far_apart(stride):
    """40 rows 2^26 elements apart: offsets pass 2^31 elements and 2^32 bytes, on 16-byte boundaries and off them."""
    g = gen(30)
    buffer = torch.zeros(40 * stride, dtype=BF16, device="cuda")
    far = lambda t: buffer.as_strided(t.shape, (stride, 1)).copy_(t)                       # noqa: E731
    x, w, r = rand(g, 40, 72, dtype=BF16), rand(g, 56, 72, dtype=BF16), rand(g, 40, 56, dtype=BF16)
    for rows in (12, 40):                                                                  # both kernels
        assert torch.equal(api.linear_forward(far(x)[:rows], w), api.linear_forward(x[:rows].contiguous(), w))
    want = api.linear_forward(x, w, residual=r)
    assert torch.equal(api.linear_forward(x, w, residual=far(r)), want)
    assert torch.equal(api.linear_forward(x, w, residual=r, out=buffer.as_strided((40, 56), (stride, 1))), want)
    assert torch.equal(api.linear_forward(w, far(x)), api.linear_forward(w, x))
    got = api.linear_backward(far(r), x, w)
    assert all(torch.equal(a, b) for a, b in zip(got, api.linear_backward(r, x, w)))
    got = api.linear_backward(r, far(x), w, r, "relu", dx=torch.empty_like(x))
    assert all(torch.equal(a, b) for a, b in zip(got, api.linear_backward(r, x, w, r, "relu")))
    y, mean, rstd = api.layer_norm_forward(x)
    near = dict(rtol=2.0 ** -7, atol=1e-5)
    assert torch.allclose(api.layer_norm_forward(far(x))[0], y, **near)
    assert torch.allclose(api.layer_norm_forward(x, out=buffer.as_strided((40, 72), (stride, 1)))[0], y, **near)
    dx, dg, db = api.layer_norm_backward(y, x, None, mean, rstd)
    for got in (api.layer_norm_backward(far(y), x, None, mean, rstd), api.layer_norm_backward(y, far(x), None, mean, rstd),
                api.layer_norm_backward(y, x, None, mean, rstd, dx=buffer.as_strided((40, 72), (stride, 1)))):
        assert torch.allclose(got[0], dx, rtol=2.0 ** -7, atol=1e-4) and torch.allclose(got[1], dg, rtol=1e-5, atol=1e-4)
    assert torch.equal(api.orthogonalize(far(x)), api.orthogonalize(x))
    assert torch.equal(api.orthogonalize(x, out=buffer.as_strided((40, 72), (stride, 1))), api.orthogonalize(x))


@pytest.mark.gpu
def test_more_than_two_to_the_31_outputs():
    """140000 x 16000 outputs and as many elements in a layer norm; rows from the beginning, the middle and the end."""
    g = gen(31)
    x, w = rand(g, 140000, 64, dtype=BF16), rand(g, 16000, 64, scale=0.1, dtype=BF16)
    y = api.linear_forward(x, w, activation="relu")
    n, mean, rstd = api.layer_norm_forward(y)
    for at in (0, 70000, 134215, 139900):                                                  # 134218 x 16000 is 2^31
        part = slice(at, at + 100)
        z, slack = products(x[part], w)
        within(y[part], act64(z, "relu"), slack, BF16)
        m64, r64, xh = norm64(y[part], 1e-5)
        assert torch.allclose(n[part].double(), xh, rtol=2.0 ** -8, atol=1e-4) and torch.allclose(rstd[part].double(), r64, rtol=1e-5)


# ---- streams, graphs, scratch, waits ------------------------------------------------------------------------------

@pytest.mark.gpu
def test_operators_on_another_stream_and_in_a_graph():
    g = gen(9)
    x, w, r = rand(g, 200, 136, dtype=BF16), rand(g, 330, 136, dtype=BF16), rand(g, 64, 100)
    dy = rand(g, 200, 330, dtype=BF16)

    def everything(stream=None):
        pre = torch.empty((200, 330), dtype=BF16, device="cuda")
        y = api.linear_forward(x, w, activation="gelu", pre=pre, stream=stream)
        n, mean, rstd = api.layer_norm_forward(y, stream=stream)
        d = api.layer_norm_backward(dy, y, None, mean, rstd, stream=stream)
        return [y, n, *d, *api.linear_backward(d[0], x, w, pre, "gelu", stream=stream), api.orthogonalize(r, stream=stream)]

    want = everything()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        inside = everything()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, inside))
    t = torch.cuda.Stream()
    t.wait_stream(torch.cuda.current_stream())
    y = api.linear_forward(x, w, activation="gelu", stream=t)
    o = api.orthogonalize(r, stream=t)
    t.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(o, want[-1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = everything()
    for _ in range(2):
        for v in out:
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.gpu
def test_scratch_is_enough_and_nothing_else_is_written():
    """Scratch and outputs inside one canary-filled buffer: exactly what the query asks for, guard bytes intact."""
    g = gen(10)
    x, w, dy, pre = (rand(g, *s, dtype=BF16) for s in ((77, 131), (65, 131), (77, 65), (77, 65)))
    m = rand(g, 2, 50, 70)
    asked = []

    def carve(need):
        big = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        asked.append((big, need))
        return big[1024:1024 + need]

    def run(call, need):
        call(carve(need))
        torch.cuda.synchronize()
        big, n = asked[-1]
        assert bool((big[:1024] == 0xA5).all()) and bool((big[1024 + n:] == 0xA5).all())
        with pytest.raises(api.RedistError) as e:
            call(carve(need)[:need - 1])
        assert e.value.status == 5

    own = api._operators()
    real = own.strided
    sizes = []
    try:
        def empty(*a, **k):                                              # what the binding allocates for itself
            if k.get("dtype") == torch.uint8:
                sizes.append(a[0][0])
            return real(*a, **k)
        own.strided = empty
        api.linear_forward(x, w)
        api.linear_backward(dy, x, w, pre, "silu")
        api.layer_norm_backward(x, x, None, torch.zeros(77, device="cuda"), torch.ones(77, device="cuda"))
        api.orthogonalize(m)
    finally:
        own.strided = real
    assert len(sizes) == 4
    run(lambda s: api.linear_forward(x, w, scratch=s), sizes[0])
    run(lambda s: api.linear_backward(dy, x, w, pre, "silu", scratch=s), sizes[1])
    run(lambda s: api.layer_norm_backward(x, x, None, torch.zeros(77, device="cuda"), torch.ones(77, device="cuda"), scratch=s), sizes[2])
    run(lambda s: api.orthogonalize(m, scratch=s), sizes[3])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,n", [(700, 640, 600), (2048, 1024, 2304), (300, 4096, 200)])
def test_a_wait_that_runs_out_is_counted_and_returns(rows, k, n):
    """test_extra_tx announces bytes that never come: every stage's wait runs out, the call returns, the counter says
    so, and the next call works.  (The copies themselves all land, so nothing is left in flight.)  Single SMs, pairs, and a
    split sum."""
    g = gen(11)
    x, w = rand(g, rows, k, dtype=BF16), rand(g, n, k, dtype=BF16)
    want = api.linear_forward(x, w)
    before = api.redist_product_timeouts()
    with api.tuning(test_extra_tx=16, wait_polls=64):
        api.linear_forward(x, w)
        torch.cuda.synchronize()
    after = api.redist_product_timeouts()
    assert after > before
    assert torch.equal(api.linear_forward(x, w), want)
    assert api.redist_product_timeouts() == after


@pytest.mark.gpu
@pytest.mark.parametrize("rows,k,n,long", [(700, 640, 600, False), (8192, 1024, 4096, True), (300, 4096, 200, False), (64, 200000, 64, True)])
def test_a_healthy_call_that_runs_out_of_polls_ends_in_order(rows, k, n, long):
    """With a handful of polls a wait runs out while copies and products are on their way, at least where a tile's sum
    takes longer than a poll (the hardware may hold a thread for microseconds in one): on the pairs that 512 full
    tiles take, and in a split sum of 200000.  The call returns; it has been counted, or its result is right; and what it
    left behind (barriers, tensor memory) does not reach the next call."""
    g = gen(13)
    x, w = rand(g, rows, k, dtype=BF16), rand(g, n, k, dtype=BF16)
    want = api.linear_forward(x, w)
    before = first = api.redist_product_timeouts()
    for polls in (1, 1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 64):
        with api.tuning(wait_polls=polls):
            got = api.linear_forward(x, w)
        after = api.redist_product_timeouts()
        assert after > before or torch.equal(got, want), polls
        assert torch.equal(api.linear_forward(x, w), want), polls
        assert api.redist_product_timeouts() == after, polls
        before = after
    assert after > first or not long                         # some of them did run out


@pytest.mark.gpu
def test_the_wait_for_a_long_sum_grows_with_it():
    """Sums of 2^22 take longer (10 ms in one piece, 0.6 ms in each of sixteen) than the polls given (1 ms, 1/4 ms), which are
    plenty for everything that does not grow with the sum."""
    g = gen(14)
    k = 1 << 22
    x = rand(g, 8, k, dtype=BF16)
    want = api.orthogonalize(x, steps=1)
    exact = orthogonalize64(x, steps=1)
    assert float((want.double() - exact).norm() / exact.norm()) < ORTHOGONAL
    before = api.redist_product_timeouts()
    with api.tuning(wait_polls=256):
        got = api.orthogonalize(x, steps=1)
    assert api.redist_product_timeouts() == before and torch.equal(got, want)
    x = rand(g, 40, k, dtype=BF16)
    want = api.linear_forward(x, x[:8])
    z, slack = products(x, x[:8])
    within(want, z, slack, BF16)
    with api.tuning(wait_polls=64):
        got = api.linear_forward(x, x[:8])
    assert api.redist_product_timeouts() == before and torch.equal(got, want)


@pytest.mark.gpu
def test_autograd_sees_what_is_written_and_nothing_else():
    """Results are not part of a graph; a tensor that is written has another version, so that a graph which kept its old
    contents says so instead of using the new ones."""
    g = gen(15)
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")               # noqa: E731
    x, w = rand(g, 40, 64, dtype=BF16).requires_grad_(), rand(g, 72, 64, dtype=BF16).requires_grad_()
    y, pre, out = api.linear_forward(x, w), z(40, 72), z(40, 72)
    assert not y.requires_grad and x._version == 0 and w._version == 0
    wide = z(40, 144)
    dx, dw, db, norm, dn, orth = z(40, 64), z(72, 64), z(72, dtype=F32), z(40, 64), z(40, 64), z(40, 64)
    xd, wd = x.detach(), w.detach()
    for call, written in ((lambda: api.linear_forward(xd, wd, out=out, pre=pre), (out, pre)),
                          (lambda: api.linear_forward(xd, wd, out=wide[:, 72:]), (wide,)),
                          (lambda: api.linear_backward(y, xd, wd, dx=dx, dw=dw, dbias=db), (dx, dw, db)),
                          (lambda: api.layer_norm_forward(xd, out=norm), (norm,)),
                          (lambda: api.layer_norm_backward(xd, xd, None, z(40, dtype=F32), z(40, dtype=F32), dx=dn), (dn,)),
                          (lambda: api.orthogonalize(xd, out=orth), (orth,))):
        before = [t._version for t in written]
        call()
        assert all(t._version > b for t, b in zip(written, before))
        assert xd._version == 0 and wd._version == 0
    leaf = torch.ones_like(out).requires_grad_()
    loss = (leaf * out).sum()                                            # keeps `out`
    api.linear_forward(xd, wd, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        api.linear_forward(xd, wd, out=torch.empty_like(out))


# ---- refusals (no GPU) ----------------------------------------------------------------------------------------------

def linear_op(**kw):
    f = dict(rows=8, in_features=16, out_features=24, type=0, bias_type=0, activation=0, reserved=0, x=(0x10000, 16, 1), w=(0x20000, 16, 1),
             residual=(None, 0, 0), out=(0x30000, 24, 1), pre=(None, 0, 0), bias=None)
    f.update(kw)
    return api._Linear(*f.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 1), (dict(in_features=0), 1), (dict(out_features=0), 1), (dict(type=2), 1), (dict(type=-1), 1), (dict(activation=4), 1),
    (dict(reserved=1), 1), (dict(x=(None, 16, 1)), 1), (dict(w=(None, 16, 1)), 1), (dict(out=(None, 24, 1)), 1), (dict(x=(0x10000, 15, 1)), 1),
    (dict(x=(0x10000, 32, 2)), 1), (dict(x=(0x10000, -16, 1)), 1), (dict(x=(0x10000, 0, 1)), 1), (dict(out=(0x30000, 1, 8)), 1),
    (dict(out=(0x30000, 23, 1)), 1), (dict(x=(0x10001, 16, 1)), 7), (dict(out=(0x30001, 24, 1)), 7), (dict(bias=0x40001), 7),
    (dict(bias=0x40000, bias_type=7), 1), (dict(out=(0x10010, 24, 1)), 6), (dict(pre=(0x30010, 24, 1)), 6), (dict(residual=(0x30010, 24, 1)), 6),
    (dict(bias=0x30010), 6), (dict(rows=1 << 31), 10), (dict(out_features=1 << 31, out=(0x30000, 1 << 31, 1)), 10),
    (dict(rows=40, x=(0x10002, 16, 1), out=(0x30000, 24, 1)), 5),          # (a few rows need no scratch)
])
def test_linear_refusals(change, status):
    assert api.load().redist_linear_forward(linear_op(**change), None, 0, None) == status


@pytest.mark.parametrize("op,grads,status", [
    (dict(), dict(dy=(None, 24, 1)), 1), (dict(), dict(dy=(0x40000, 1, 8)), 1), (dict(activation=2), dict(), 1),
    (dict(), dict(dx=(0x50000, 15, 1)), 1), (dict(), dict(dw=(0x60000, 15, 1)), 1), (dict(), dict(dx=(0x10000, 16, 1)), 6),
    (dict(), dict(dw=(0x50000, 16, 1)), 6), (dict(), dict(dbias=0x60000), 6), (dict(), dict(dbias=0x70002), 7), (dict(), dict(dbias=0x70000), 5),
    (dict(activation=1, pre=(0x80000, 24, 1)), dict(), 5), (dict(w=(None, 0, 0)), dict(), 1), (dict(x=(None, 0, 0)), dict(), 1),
])
def test_linear_backward_refusals(op, grads, status):
    f = dict(dy=(0x40000, 24, 1), dx=(0x50000, 16, 1), dw=(0x60000, 16, 1), dbias=None)
    f.update(grads)
    assert api.load().redist_linear_backward(linear_op(out=(None, 0, 0), **op), api._LinearGrads(*f.values()), None, 0, None) == status


def norm_op(**kw):
    f = dict(rows=4, cols=32, type=2, weight_type=2, eps=1e-5, reserved=0, x=(0x10000, 32, 1), y=(0x20000, 32, 1), gamma=None, beta=None,
             mean=0x30000, rstd=0x31000)
    f.update(kw)
    return api._LayerNorm(*f.values())


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 1), (dict(cols=0), 1), (dict(eps=-1.0), 1), (dict(eps=float("nan")), 1), (dict(type=3), 1), (dict(gamma=0x40000, weight_type=3), 1),
    (dict(reserved=2), 1), (dict(x=(None, 32, 1)), 1), (dict(x=(0x10000, 31, 1)), 1), (dict(x=(0x10000, 1, 4)), 1), (dict(y=(None, 32, 1)), 1),
    (dict(y=(0x20002, 32, 1)), 7), (dict(x=(0x10002, 32, 1)), 7), (dict(gamma=0x40002), 7), (dict(mean=0x30002), 7), (dict(y=(0x10000, 32, 1)), 6),
    (dict(mean=0x20000), 6), (dict(gamma=0x20000), 6), (dict(rstd=0x30000), 6), (dict(cols=1 << 31, x=(0x10000, 1 << 31, 1)), 10),
])
def test_layer_norm_refusals(change, status):
    assert api.load().redist_layer_norm_forward(norm_op(**change), None) == status


@pytest.mark.parametrize("change,grads,status", [
    (dict(mean=None), dict(), 1), (dict(rstd=None), dict(), 1), (dict(), dict(dy=(None, 32, 1)), 1), (dict(), dict(dx=(0x10000, 32, 1)), 6),
    (dict(), dict(dgamma=0x70000), 6), (dict(), dict(dgamma=0x80002), 7), (dict(), dict(dgamma=0x80000), 5),
])
def test_layer_norm_backward_refusals(change, grads, status):
    f = dict(dy=(0x60000, 32, 1), dx=(0x70000, 32, 1), dgamma=None, dbeta=None)
    f.update(grads)
    assert api.load().redist_layer_norm_backward(norm_op(**change), api._LayerNormGrads(*f.values()), None, 0, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), 1), (dict(rows=0), 1), (dict(cols=0), 1), (dict(steps=0), 1), (dict(steps=65), 1), (dict(type=3), 1), (dict(eps=0.0), 1),
    (dict(eps=float("nan")), 1), (dict(scale=float("inf")), 1), (dict(reserved=1), 1), (dict(x=(None, 32, 1)), 1), (dict(x=(0x10000, 31, 1)), 1),
    (dict(x=(0x10000, 1, 16)), 1), (dict(out=(0x90000, 1, 16)), 1), (dict(out=(0x90001, 32, 1)), 7), (dict(x=(0x10001, 32, 1)), 7),
    (dict(out_batch_stride=511), 1), (dict(batch=70000), 10), (dict(coefficients=None), 1), (dict(out=(0x10000, 32, 1)), 6), (dict(), 5),
    (dict(abc=(100.0, 0.0, 0.0)), 1), (dict(abc=(float("nan"), 0.0, 0.0)), 1), (dict(x_batch_stride=-1), 1),
])
def test_orthogonalize_refusals(change, status):
    change = dict(change)
    abc = (ctypes.c_float * (3 * 64))(*(list(change.pop("abc", MUON)) * 64))
    f = dict(batch=2, rows=16, cols=32, type=0, steps=5, eps=1e-7, scale=1.0, reserved=0, x=(0x10000, 32, 1), out=(0x90000, 32, 1),
             x_batch_stride=512, out_batch_stride=512, coefficients=ctypes.addressof(abc))
    f.update(change)
    assert api.load().redist_orthogonalize(api._Orthogonal(*f.values()), None, 0, None) == status


def test_null_arguments_are_refused():
    lib = api.load()
    assert lib.redist_linear_forward(None, None, 0, None) == 1 and lib.redist_linear_backward(None, None, None, 0, None) == 1
    assert lib.redist_layer_norm_forward(None, None) == 1 and lib.redist_layer_norm_backward(None, None, None, 0, None) == 1
    assert lib.redist_orthogonalize(None, None, 0, None) == 1
    assert lib.redist_linear_scratch_bytes(None, None) == 0 and lib.redist_layer_norm_scratch_bytes(None, None) == 0
    assert lib.redist_orthogonalize_scratch_bytes(None) == 0


def test_the_binding_refuses_before_the_foreign_call():
    x, w = torch.zeros((4, 8), dtype=BF16), torch.zeros((6, 8), dtype=BF16)
    for call in (lambda: api.linear_forward(x, w), lambda: api.linear_backward(torch.zeros((4, 6), dtype=BF16), x, w),
                 lambda: api.layer_norm_forward(x), lambda: api.layer_norm_backward(x, x, None, torch.zeros(4), torch.zeros(4)),
                 lambda: api.orthogonalize(x), lambda: api.linear_forward(x[0], w), lambda: api.orthogonalize(x, steps=0),
                 lambda: api.orthogonalize(x, coefficients=(1.0, 2.0))):
        with pytest.raises(api.RedistError) as e:
            call()                                                       # host tensors, vectors, wrong options
        assert e.value.status == 1


class ScratchElsewhere:
    """A scratch tensor on another device than the operands, as far as the binding looks at one."""
    is_cuda, device = True, torch.device("cuda", 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x1000000

    def numel(self):
        return 1 << 20

    def element_size(self):
        return 1


def test_scratch_on_another_device_is_refused():
    o = api._operators()
    assert o.scratch(256, ScratchElsewhere(), torch.device("cuda", 1))[1:] == (0x1000000, 1 << 20)
    with pytest.raises(api.RedistError) as e:
        o.scratch(256, ScratchElsewhere(), torch.device("cuda", 0))
    assert e.value.status == 1


@pytest.mark.gpu
def test_the_binding_refuses_mismatched_tensors():
    z = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")               # noqa: E731
    x, w = z(4, 8), z(6, 8)
    for call in (lambda: api.linear_forward(x, z(6, 9)), lambda: api.linear_forward(x, z(6, 8, dtype=F16)), lambda: api.linear_forward(x, w.cpu()),
                 lambda: api.linear_forward(x, w, bias=z(5)), lambda: api.linear_forward(x, w, bias=z(12)[::2]),
                 lambda: api.linear_forward(x, w, bias=z(6, dtype=torch.float64)), lambda: api.linear_forward(x, w, residual=z(4, 5)),
                 lambda: api.linear_forward(x, w, out=z(4, 6, dtype=F32)), lambda: api.linear_forward(x, w, activation="tanh"),
                 lambda: api.linear_forward(z(4, 8, dtype=F32), z(6, 8, dtype=F32)), lambda: api.linear_forward(z(4, 16)[:, ::2], w),
                 lambda: api.linear_forward(z(1, 8).expand(4, 8), w),
                 lambda: api.linear_backward(z(4, 6), x, w, activation="gelu"), lambda: api.linear_backward(z(4, 5), x, w),
                 lambda: api.linear_backward(z(6, 4).T, x, w),
                 lambda: api.layer_norm_forward(z(8, 4).T), lambda: api.layer_norm_forward(x, gamma=z(7)),
                 lambda: api.layer_norm_forward(x, z(8), z(8, dtype=F32)), lambda: api.layer_norm_forward(x, out=z(4, 8, dtype=F16)),
                 lambda: api.layer_norm_backward(x, x, None, z(4), z(4)), lambda: api.layer_norm_backward(x, z(4, 9), None, z(4, dtype=F32), z(4, dtype=F32)),
                 lambda: api.orthogonalize(x, out=z(4, 8, dtype=F16)), lambda: api.orthogonalize(z(8, 4).T), lambda: api.orthogonalize(z(4)),
                 lambda: api.orthogonalize(x, coefficients=(50.0, 0.0, 0.0)), lambda: api.orthogonalize(z(4, 8, dtype=torch.float64))):
        with pytest.raises(api.RedistError) as e:
            call()
        assert e.value.status == 1
