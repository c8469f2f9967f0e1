"""Products that run for a large part of a second: nothing in a kernel waits as long as the whole of it takes.

Tolerances as in the tests of the linear layer: a sum of k products in 32 bits is off by at most (k + 2) 2^-23 of the sum of
their magnitudes, an output by half a unit of its type.
"""
import pytest

from paper_2112_01075_b200 import api
from test_operators import BF16, gen, products, within

torch = pytest.importorskip("torch")

N = 1 << 16


@pytest.fixture(scope="module")
def operands():
    """131072 x 65536 and 65536 x 65536: 26 GB, and a product of them takes 0.8 s (2^50 operations)."""
    g = gen(1)
    x, w = (torch.empty((rows, N), dtype=BF16, device="cuda").normal_(generator=g) for rows in (2 * N, N))
    yield x, w.mul_(N ** -0.5)


def check(x, w, y):
    rows = torch.tensor([0, 1, 127, 128, 20000, 40001, y.shape[0] - 1], device="cuda")
    cols = torch.tensor([0, 255, 256, 30000, 50021, 65535], device="cuda")
    z, slack = products(x[rows], w[cols])
    within(y[rows][:, cols], z, slack, BF16)
    assert bool(torch.isfinite(y[::97, ::89]).all())


@pytest.mark.gpu
def test_a_long_product_is_not_counted_as_one_that_waited_in_vain(operands):
    x, w = operands
    before = api.redist_product_timeouts()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    y = api.linear_forward(x, w)
    end.record()
    assert api.redist_product_timeouts() == before
    assert start.elapsed_time(end) > 600, "hardly longer than the limit of a wait for products that have been issued"
    check(x, w, y)


@pytest.mark.gpu
def test_a_long_product_by_expert_is_not_counted_as_one_that_waited_in_vain(operands):
    x, w = operands
    before = api.redist_product_timeouts()
    offsets = torch.tensor([0, 2 * N], dtype=torch.int32, device="cuda")
    y = api.experts_forward(x, w[None], offsets)
    assert api.redist_product_timeouts() == before
    check(x, w, y)
    del y
    dy = torch.empty_like(x).normal_(generator=gen(2))
    _, dw, _ = api.experts_backward(dy, x, w[None], offsets, need=(False, True, False))
    assert api.redist_product_timeouts() == before
    check(dy.T, x.T, dw[0])
