"""Every tile shape of the operators' matrix products, at sizes that are ragged for it: what large calls run on.

The shape that a call takes follows from its size, and small calls take few of them; the tuning values
"test_product_shape" and "test_product_parts" force the others.  Tolerances are test_operators.py's."""
import pytest

from paper_2112_01075_b200 import api

torch = pytest.importorskip("torch")

import test_operators as T                                                            # noqa: E402
from test_operators import BF16, F16, F32, gen, no_wait_runs_out, products, rand, within   # noqa: E402,F401

SHAPES = {1: "256x256 pair", 2: "256x128 pair", 3: "128x256", 4: "128x128", 5: "128x64"}
PARTS = (1, 3)
every_shape = pytest.mark.parametrize("shape", SHAPES, ids=SHAPES.get)


def test_the_values_have_their_documented_default_and_range():
    for name, hi in (("test_product_shape", 5), ("test_product_parts", 16)):
        assert api.tuning_get(name) == 0
        for bad in (-1, hi + 1):
            with pytest.raises(api.RedistError):
                api.tuning_set(name, bad)
        with api.tuning(**{name: hi}):
            assert api.tuning_get(name) == hi
        assert api.tuning_get(name) == 0


def inside(t, left, right):
    """``t`` as a block of columns of a wider matrix that is otherwise NaN."""
    big = torch.full((t.shape[0], left + t.shape[1] + right), float("nan"), dtype=t.dtype, device="cuda")
    view = big[:, left:left + t.shape[1]]
    view.copy_(t)
    return view


def columns_first(t):
    return t.T.contiguous().T


class Framed:
    """An output inside a wider and taller matrix; what surrounds it has to stay."""

    def __init__(self, rows, cols, dtype, left, right):
        self.big = torch.full((rows + 2, left + cols + right), 7.0, dtype=dtype, device="cuda")
        self.view = self.big[1:rows + 1, left:left + cols]
        self.view.fill_(float("nan"))

    def check(self):
        rest = self.big.clone()
        r, c = self.view.shape
        at = self.view.storage_offset() % self.big.shape[1]
        rest[1:r + 1, at:at + c] = 7.0
        assert bool((rest == 7.0).all())


@pytest.mark.gpu
@every_shape
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("rows,k,n,left", [(385, 520, 328, 8), (299, 331, 517, 1), (40, 1000, 263, 0), (260, 72, 24, 3)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_forward(shape, parts, rows, k, n, left, dtype):
    """Both orders of both operands; bias, pre-activation, activation and residual, on 16-byte boundaries and off them."""
    g = gen(shape * 100 + rows)
    x, w, residual = rand(g, rows, k, dtype=dtype), rand(g, n, k, scale=k ** -0.5, dtype=dtype), rand(g, rows, n, dtype=dtype)
    bias = rand(g, n)
    z, slack = products(x, w)
    zb = z + bias.double()
    slack_b = slack + 2.0 ** -23 * zb.abs()
    with api.tuning(test_product_shape=shape, test_product_parts=parts):
        for i, (ox, ow) in enumerate(((0, 0), (0, 1), (1, 0), (1, 1))):
            xx, ww = (columns_first(x) if ox else x), (columns_first(w) if ow else inside(w, left, 8))
            out = Framed(rows, n, dtype, left, 8)
            api.linear_forward(xx, ww, out=out.view)
            within(out.view, z, slack, dtype)
            out.check()
            activation = api.ACTIVATIONS[i]
            out, pre = Framed(rows, n, dtype, left, 8), Framed(rows, n, dtype, left, 8)
            api.linear_forward(xx, ww, bias, inside(residual, left, 5), activation, out=out.view, pre=pre.view)
            within(pre.view, zb, slack_b, dtype)
            want = T.act64(zb, activation) + residual.double()
            within(out.view, want, slack_b * T.STEEPEST[activation] + 2.0 ** -20 * (zb.abs() + want.abs()), dtype)
            out.check()
            pre.check()
        over = residual.clone()                                                       # the residual itself as output
        api.linear_forward(x, w, residual=over, out=over)
        within(over, z + residual.double(), slack + 2.0 ** -23 * (z + residual.double()).abs(), dtype)


@pytest.mark.gpu
@every_shape
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("rows,k,n,left", [(400, 264, 328, 8), (299, 331, 517, 1)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_backward(shape, parts, rows, k, n, left, dtype):
    g = gen(shape * 100 + rows + 1)
    x, w = rand(g, rows, k, dtype=dtype), rand(g, n, k, scale=k ** -0.5, dtype=dtype)
    pre, dy = rand(g, rows, n, dtype=dtype), rand(g, rows, n, dtype=dtype)
    wa, xa = w.double().abs(), x.double().abs()
    for activation in ("none", "gelu"):
        dz = dy.double() * T.slope64(pre.double(), activation)
        off = dz.abs() * T.HALF_ULP[dtype] * (activation != "none") + dy.double().abs() * 2.0 ** -20 + T.TINY[dtype]
        for xx, ww in ((x, w), (columns_first(x), columns_first(w))):
            dx, dw = Framed(rows, k, dtype, left, 8), Framed(n, k, dtype, left, 8)
            with api.tuning(test_product_shape=shape, test_product_parts=parts):
                _, _, db = api.linear_backward(inside(dy, left, 8), xx, ww, inside(pre, left, 8), activation, dx=dx.view, dw=dw.view)
            within(dx.view, dz @ w.double(), off @ wa + (n + 2) * 2.0 ** -23 * (dz.abs() @ wa), dtype)
            within(dw.view, dz.T @ x.double(), off.T @ xa + (rows + 2) * 2.0 ** -23 * (dz.abs().T @ xa), dtype)
            within(db, dz.sum(0), (dy.double().abs() * 2.0 ** -20).sum(0) + (rows + 2) * 2.0 ** -24 * dz.abs().sum(0), F32)
            dx.check()
            dw.check()


@pytest.mark.gpu
@every_shape
@pytest.mark.parametrize("batch,m,n", [(2, 300, 700), (2, 700, 300), (1, 520, 520), (3, 129, 257), (1, 1100, 1030)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_orthogonalize(shape, batch, m, n, dtype):
    """Mirrored tiles (not on 128x256, which only the updates of X take), the mean of the diagonal, the pair of 16-bit halves,
    and outputs off 16-byte boundaries."""
    x = (T.gradient_like(gen(m + n + shape), batch, m, n, "gaussian") * 2.0 ** -7).to(dtype)
    want = T.orthogonalize64(x)
    out = torch.full((batch, m + 1, n + 5), 7.0, dtype=BF16, device="cuda")
    with api.tuning(test_product_shape=shape):
        got = api.orthogonalize(x)
        api.orthogonalize(x, out=out[:, :m, 3:n + 3])
    for i in range(batch):
        assert float((got[i].double() - want[i]).norm() / want[i].norm()) < T.ORTHOGONAL
    assert torch.equal(out[:, :m, 3:n + 3], got)
    assert bool((out[:, m] == 7).all()) and bool((out[..., :3] == 7).all()) and bool((out[..., n + 3:] == 7).all())


@pytest.mark.gpu
@every_shape
@pytest.mark.parametrize("parts", PARTS)
def test_a_wait_that_runs_out_returns(shape, parts):
    """test_extra_tx announces bytes that never come, on every shape; and a few polls for healthy calls of long sums."""
    g = gen(16)
    x, w = rand(g, 300, 4000, dtype=BF16), rand(g, 520, 4000, dtype=BF16)
    m = rand(g, 2, 300, 4000)
    # what the next call gives: a sum's order is the shape's and the parts'
    with api.tuning(test_product_shape=shape, test_product_parts=parts):
        want, orthogonal = api.linear_forward(x, w), api.orthogonalize(m)
    before = api.redist_product_timeouts()
    with api.tuning(test_product_shape=shape, test_product_parts=parts, test_extra_tx=16, wait_polls=64):
        api.linear_forward(x, w)
        api.orthogonalize(m)
    after = api.redist_product_timeouts()
    assert after > before
    for polls in (1, 2, 3, 5, 8):
        before = after
        with api.tuning(test_product_shape=shape, test_product_parts=parts, wait_polls=polls):
            first, second = api.linear_forward(x, w), api.orthogonalize(m)
        after = api.redist_product_timeouts()
        assert after > before or (torch.equal(first, want) and torch.equal(second, orthogonal)), polls
    with api.tuning(test_product_shape=shape, test_product_parts=parts):
        assert torch.equal(api.linear_forward(x, w), want) and torch.equal(api.orthogonalize(m), orthogonal)
    assert api.redist_product_timeouts() == after


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 5, 8, 9, 16, 17, 20, 32])
@pytest.mark.parametrize("k,n", [(4097, 77), (4097, 130), (8200, 200), (16400, 65)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_few_rows_with_a_sum_split_over_a_cluster(rows, k, n, dtype):
    """The kernel of a few rows, on 16-byte boundaries and off them, with sums long enough for two to eight blocks."""
    g = gen(rows + k + n)
    x, w, residual = rand(g, rows, k, dtype=dtype), rand(g, n, k, scale=k ** -0.5, dtype=dtype), rand(g, rows, n, dtype=dtype)
    bias = rand(g, n, dtype=dtype)
    z, slack = products(x, w)
    z = z + bias.double()
    slack = slack + 2.0 ** -23 * z.abs()
    for left in (0, 1, 8):
        out, pre = Framed(rows, n, dtype, left, 3), Framed(rows, n, dtype, left, 3)
        api.linear_forward(inside(x, left, 8), inside(w, left, 8), bias, inside(residual, left, 3), "silu", out=out.view, pre=pre.view)
        within(pre.view, z, slack, dtype)
        want = T.act64(z, "silu") + residual.double()
        within(out.view, want, slack * T.STEEPEST["silu"] + 2.0 ** -20 * (z.abs() + want.abs()), dtype)
        out.check()
        pre.check()
