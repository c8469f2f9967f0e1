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
