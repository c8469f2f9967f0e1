"""The bound on a step's gradients where 32 bits do not hold the norm, or the factor: the tensors are finite, so is what the formula
gives, min(1, max_norm / (|g| + eps)) g.

The norm is off by (65 / 2 + 1) 2^-24 of itself and the factor by four roundings more, as in the other tests of it; below 2^-126 an
output is off by half a subnormal step besides.
"""
import math

import pytest

from paper_2112_01075_b200 import api
from test_operators import BF16, F16, F32, gen, rand, within

torch = pytest.importorskip("torch")

INF = math.inf
OFF = (65 / 2 + 5) * 2.0 ** -24


def clipped(tensors, bound, eps=1e-6):
    total = math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))
    return [t.double() * min(1.0, bound / (total + eps)) for t in tensors], total


@pytest.mark.gpu
@pytest.mark.parametrize("bound", [3e38, 1e38, 1e30, 1.0, 1e-10, 1e-38, 0.0, INF])
@pytest.mark.parametrize("size", [3e38, 1e38, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norms_beyond_32_bits(size, bound, dtype):
    g = gen(1)
    keep = [(torch.rand(n, generator=g, device="cuda") * size).to(dtype) for n in (5000, 3, 700)]
    want, total = clipped(keep, bound)
    for given in (False, True):
        tensors = [t.clone() for t in keep]
        out = [torch.full_like(t, 7.0) for t in keep] if given else None
        norm = float(api.clip_gradients(tensors, bound, out=out))
        assert norm == INF if total > 3.41e38 else abs(norm - total) <= OFF * total
        for a, b in zip(out if given else tensors, want):
            within(a, b, b.abs() * OFF + 2.0 ** -149, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_factors_beyond_32_bits(dtype):
    """Bounds so small that the quotient is subnormal, or less, in 32 bits: gradients below that then, but not cut to what its few
    bits say."""
    g = gen(2)
    keep = [rand(g, 4000, dtype=dtype), rand(g, 60, dtype=dtype)]
    for scale, bound in ((1.0, 1e-37), (2.0 ** 12, 1e-36), (2.0 ** 12, 3e-38)):
        tensors = [(t.float() * scale).to(dtype) for t in keep]
        want, _ = clipped(tensors, bound)
        api.clip_gradients(tensors, bound)
        for a, b in zip(tensors, want):
            within(a, b, b.abs() * OFF + 2.0 ** -149, dtype)


@pytest.mark.gpu
def test_infinities_and_nan_stay_what_they_are():
    for bad in (INF, math.nan):
        a, b = torch.tensor([1.0, bad, 3e38], device="cuda"), torch.full((500,), 3e38, device="cuda")
        api.clip_gradients([a, b], 1.0)
        if bad == INF:
            assert a[0] == 0 and bool(torch.isnan(a[1])) and a[2] == 0 and not bool(b.any())
        else:
            assert bool(torch.isnan(a).all()) and bool(torch.isnan(b).all())
    a = torch.zeros(10, device="cuda")
    assert float(api.clip_gradients([a], 0.0)) == 0 and not bool(a.any())
