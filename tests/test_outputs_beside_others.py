"""Outputs whose rows start on 16-byte boundaries and end within 16 bytes, inside larger arrays: what lies behind a row's end stays.

A tensor store of the TMA writes whole 16 bytes, and so must not be used for the end of such a row.
"""
import pytest

from paper_2112_01075_b200 import api
from test_experts_variants import Guarded, ranges
from test_operators import BF16, F16, F32, HALF_ULP, TINY, gen, products, rand, slope64, within

torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def no_wait_runs_out(request):
    before = api.redist_product_timeouts() if "gpu" in request.keywords else 0
    yield
    assert "gpu" not in request.keywords or api.redist_product_timeouts() == before


def room(*shape, dtype, more=0, apart=0):
    """Rows 8, 16, ... elements apart that have room behind them; matrices `apart` rows further."""
    return Guarded(*shape, dtype=dtype, extra=-shape[-1] % 8 + 8 * more, apart=apart)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [0, 1, 2, 3, 4, 5])
@pytest.mark.parametrize("counts,before,behind,k,n", [
    ([40, 0, 130, 64], 0, 0, 72, 35), ([300, 33], 2, 3, 96, 270), ([64, 200, 31, 1], 0, 5, 100, 513), ([500], 0, 0, 41, 127), ([70] * 9, 1, 0, 33, 1),
    ([96, 64], 0, 0, 1, 100), ([33, 64, 0, 5], 0, 0, 260, 7),
])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_products_by_expert(counts, before, behind, k, n, shape, dtype):
    offsets, rows, owner = ranges(counts, before, behind)
    used, e, g = owner >= 0, len(counts), gen(sum(counts) + k + n)
    x, w = rand(g, rows, k, dtype=dtype), rand(g, e, n, k, scale=k ** -0.5, dtype=dtype)
    pre, dy = rand(g, rows, n, dtype=dtype), rand(g, rows, n, dtype=dtype)
    for more, apart in ((0, 0), (1, 1)):
        y, z = room(rows, n, dtype=dtype, more=more), room(rows, n, dtype=dtype, more=more)
        dx, dw = room(rows, k, dtype=dtype, more=more), room(e, n, k, dtype=dtype, more=more, apart=apart)
        with api.tuning(test_product_shape=shape):
            api.experts_forward(x, w, offsets, out=y.t, pre=z.t)
            api.experts_backward(dy, x, w, offsets, pre, "silu", dx=dx.t, dw=dw.t)
        assert y.intact(used) and z.intact(used) and dx.intact(used) and dw.intact()
        for i, c in enumerate(counts):
            at = (owner == i).nonzero().flatten()
            want, slack = products(x[at], w[i])
            within(y.t[at], want, slack, dtype)
            assert torch.equal(y.t[at], z.t[at])
            d, xs, wi = dy[at].double(), x[at].double(), w[i].double()
            dz = d * slope64(pre[at].double(), "silu")
            off = dz.abs() * HALF_ULP[dtype] + d.abs() * 2.0 ** -20 + TINY[dtype]
            within(dx.t[at], dz @ wi, off @ wi.abs() + (n + 2) * 2.0 ** -23 * (dz.abs() @ wi.abs()), dtype)
            within(dw.t[i], dz.T @ xs, off.T @ xs.abs() + (c + 2) * 2.0 ** -23 * (dz.abs().T @ xs.abs()), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("k", [1, 4, 20, 35, 100, 1604, 2055])
@pytest.mark.parametrize("experts", [1, 3])
def test_gradients_of_weights_of_one_row(k, experts):
    """One output feature: dw's only row has nothing behind it but what belongs to others."""
    offsets, rows, _ = ranges([70, 0, 41][:experts], 0, 0)
    g = gen(k)
    x, dy, w = rand(g, rows, k, dtype=BF16), rand(g, rows, 1, dtype=BF16), rand(g, experts, 1, k, dtype=BF16)
    for extra in (0, 3, 8 - k % 8):
        dw = Guarded(experts, 1, k, extra=extra)
        api.experts_backward(dy, x, w, offsets, need=(False, True, False), dw=dw.t)
        assert dw.intact()
        for i in range(experts):
            at = slice(int(offsets[i]), int(offsets[i + 1]))
            want, slack = products(dy[at].T.contiguous(), x[at].T.contiguous())
            within(dw.t[i], want, slack, BF16)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", range(0, 6))
@pytest.mark.parametrize("rows,k,n", [(40, 96, 35), (300, 35, 270), (700, 65, 1), (130, 1, 100), (33, 1604, 513), (1, 2055, 40), (513, 200, 7)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_linear_layers(rows, k, n, shape, dtype):
    g = gen(rows + k + n)
    x, w, r = rand(g, rows, k, dtype=dtype), rand(g, n, k, scale=k ** -0.5, dtype=dtype), rand(g, rows, n, dtype=dtype)
    pre, dy = rand(g, rows, n, dtype=dtype), rand(g, rows, n, dtype=dtype)
    z, slack = products(x, w)
    d = dy.double()
    dz = d * slope64(pre.double(), "silu")
    off = dz.abs() * HALF_ULP[dtype] + d.abs() * 2.0 ** -20 + TINY[dtype]
    for more in (0, 1):
        y, p, dx, dw = (room(*s, dtype=dtype, more=more) for s in ((rows, n), (rows, n), (rows, k), (n, k)))
        joined = room(rows, n, dtype=dtype, more=more)
        beside = room(rows, n, dtype=dtype, more=more)
        beside.t.copy_(r)
        with api.tuning(test_product_shape=shape):
            api.linear_forward(x, w, out=y.t, pre=p.t)
            api.linear_forward(x, w, residual=beside.t, out=joined.t)
            api.linear_forward(x, w, residual=beside.t, out=beside.t)
            api.linear_backward(dy, x, w, pre, "silu", dx=dx.t, dw=dw.t)
        assert all(t.intact() for t in (y, p, dx, dw, joined, beside))
        within(y.t, z, slack, dtype)
        assert torch.equal(y.t, p.t) and torch.equal(joined.t, beside.t)
        within(joined.t, z + r.double(), slack + 2.0 ** -23 * (z + r.double()).abs(), dtype)
        within(dx.t, dz @ w.double(), off @ w.double().abs() + (n + 2) * 2.0 ** -23 * (dz.abs() @ w.double().abs()), dtype)
        within(dw.t, dz.T @ x.double(), off.T @ x.double().abs() + (rows + 2) * 2.0 ** -23 * (dz.abs().T @ x.double().abs()), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,m,n", [(1, 130, 35), (1, 260, 513), (3, 64, 100), (2, 33, 7), (1, 1, 41), (2, 1, 20)])
def test_orthogonalisation(batch, m, n):
    x = rand(gen(m + n), batch, m, n, dtype=BF16)
    want = api.orthogonalize(x)
    for more, apart in ((0, 0), (1, 0), (0, 2)):
        out = room(batch, m, n, dtype=BF16, more=more, apart=apart)
        api.orthogonalize(x, out=out.t)
        assert out.intact() and torch.equal(out.t, want)
