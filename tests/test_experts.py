"""The operators of a block of experts -- router, moves of tokens to their experts' rows and back, products grouped by expert
-- and the bound on a step's gradients, against their definitions in 64 bits.

Tolerances are derived as in the tests of the linear layer: an output rounded once to a type with p significant bits is off
by 2^-p of itself, a sum of k products in 32 bits by at most k 2^-23 of the sum of their magnitudes.
"""
import ctypes
import math

import pytest

from paper_2112_01075_b200 import api
from test_operators import HALF_ULP, STEEPEST, TINY, act64, gen, products, rand, slope64, within

torch = pytest.importorskip("torch")

BF16, F16, F32, I32 = torch.bfloat16, torch.float16, torch.float32, torch.int32
INF, NAN = math.inf, math.nan


@pytest.fixture(autouse=True)
def no_wait_runs_out(request):
    """No test may leave a bounded wait behind that ran out (but the one that makes them)."""
    counts = "gpu" in request.keywords and "runs_out" not in request.node.name
    before = api.redist_product_timeouts() if counts else 0
    yield
    assert not counts or api.redist_product_timeouts() == before


# ---- router -------------------------------------------------------------------------------------------------------------

def route64(logits, k, normalize):
    """Weights, choice, position and offsets by the definition, and the relative error that 32 bits may make in a weight."""
    l = logits.double()
    n, e = l.shape
    ranked = torch.sort(l, dim=1, descending=True, stable=True)              # NaN first, ties by index
    value, choice = ranked.values[:, :k], ranked.indices[:, :k]
    some = value != -INF
    over = value if normalize else l
    top = value[:, :1]
    base = torch.exp(over - top).masked_fill(over == -INF, 0).sum(1, keepdim=True)
    weights = (torch.exp(value - top) / base).masked_fill(~some, 0.0)
    choice = choice.masked_fill(~some, -1)
    flat = torch.where(some, choice, e).reshape(-1)
    order = torch.sort(flat, stable=True).indices
    position = torch.empty_like(flat)
    position[order] = torch.arange(n * k, device=l.device)
    position = position.view(n, k).masked_fill(~some, -1)
    count = torch.bincount(flat, minlength=e + 1)[:e]
    offsets = torch.nn.functional.pad(count.cumsum(0), (1, 0))
    # exponents are off by 2^-24 of themselves, exp by 2 units (2^-22), twice; the sum of up to e terms and the quotient by 2^-24 each
    spread = (top - over.masked_fill(over == -INF, INF).amin(1, keepdim=True)).clamp(0, 104).nan_to_num(0)
    off = 2 * (spread * 2.0 ** -24 + 2.0 ** -22) + (over.shape[1] + 2) * 2.0 ** -24
    return weights, choice, position, offsets, off


ROUTES = [  # tokens, experts, k
    (0, 5, 2), (1, 1, 1), (1, 2, 2), (3, 8, 8), (16, 64, 4), (17, 9, 3), (100, 32, 32), (127, 33, 5), (128, 300, 6), (129, 200, 32), (1000, 100, 8),
    (5000, 1024, 32), (20000, 6, 2), (70001, 3, 1), (16384, 128, 8),
]


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,experts,k", ROUTES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("normalize", [True, False])
def test_route(tokens, experts, k, dtype, normalize):
    g = gen(tokens + experts * 3 + k)
    logits = rand(g, tokens, experts, scale=3.0, dtype=dtype)
    if experts > 4:                                                          # masked experts and tokens, ties, both zeros
        logits[torch.rand((tokens, experts), generator=g, device="cuda") < 0.1] = -INF
        logits[torch.rand(tokens, generator=g, device="cuda") < 0.05] = -INF
        tied = torch.rand(tokens, generator=g, device="cuda") < 0.2
        logits[tied] = logits[tied].round()
    want, choice, position, offsets, off = route64(logits, k, normalize)
    w, c, p, o = api.route_forward(logits, k, normalize=normalize)
    assert torch.equal(c, choice.int()) and torch.equal(p, position.int()) and torch.equal(o, offsets.int())
    within(w, want, want * off + 2.0 ** -126, F32)
    # the gradient: of the weights as they are, so that only its own roundings count
    dw = rand(g, tokens, k)
    dw[choice < 0] = NAN                                                     # does not count
    got = api.route_backward(dw, logits, w, c, normalize=normalize)
    d = dw.double().masked_fill(choice < 0, 0)
    part = w.double() * d
    mean = part.sum(1, keepdim=True)
    sizes = part.abs().sum(1, keepdim=True)
    at = choice.clamp(min=0)
    if normalize:
        grad = torch.zeros((tokens, experts), dtype=torch.float64, device="cuda").scatter_add(1, at, w.double() * (d - mean))
        slack = torch.zeros_like(grad).scatter_add(1, at, w.double() * (d.abs() + (k + 2) * sizes) * 2.0 ** -22)
    else:
        top = logits.double().amax(1, keepdim=True) if experts else None
        e = torch.exp(logits.double() - torch.where(top > -INF, top, 0.0))
        prob = e / e.sum(1, keepdim=True).clamp(min=1e-300)
        grad = torch.zeros_like(prob).scatter_add(1, at, part) - prob * mean
        slack = torch.zeros_like(prob).scatter_add(1, at, part.abs() * 2.0 ** -22) + prob * (off + (k + 3) * 2.0 ** -22) * sizes
    within(got, grad, slack + 2.0 ** -126, dtype)


@pytest.mark.gpu
def test_route_special_values():
    x = torch.tensor([[0.0, -0.0, 1.0, 1.0], [NAN, INF, 5.0, 1.0], [1.0, NAN, NAN, -INF], [-INF, -INF, 2.0, -INF], [-INF] * 4, [INF, INF, 0.0, 1.0],
                      [3e38, -3e38, 0.0, 1.0]], device="cuda")
    for normalize in (True, False):
        w, c, p, o = api.route_forward(x, 3, normalize=normalize)
        assert c.tolist() == [[2, 3, 0], [0, 1, 2], [1, 2, 0], [2, -1, -1], [-1, -1, -1], [0, 1, 3], [0, 3, 2]]
        assert w[3].tolist() == [1, 0, 0] and w[4].tolist() == [0, 0, 0] and bool(torch.isnan(w[1]).all()) and bool(torch.isnan(w[2]).all())
        assert bool(torch.isnan(w[5, :2]).all()) and w[6].tolist() == [1, 0, 0]
        assert o.tolist() == [0, 5, 8, 13, 16]
        rows = p[p >= 0]
        assert torch.equal(rows.sort().values, torch.arange(int(o[-1]), device="cuda", dtype=I32))
        d = api.route_backward(torch.ones((7, 3), device="cuda"), x, w, c, normalize=normalize)
        assert not bool(d[4].any()) and not bool(d[3].any()) and bool(torch.isnan(d[1, :2]).all())


@pytest.mark.gpu
def test_route_strides_and_gradient_against_differences():
    """(L(x + h v) - L(x - h v)) / 2h against <dx, v>, L = <weights, dw> in 32 bits: weights are off by about 2^-22, which is
    divided by h; central differences by h^2 / 6 of a third derivative of up to 6 |dw| |v|^3 or so."""
    g = gen(6)
    x0 = rand(g, 40, 23)
    big = torch.full((40, 31), NAN, device="cuda")
    x = big[:, 5:28]
    x.copy_(x0)
    h = 2.0 ** -6
    for normalize in (True, False):
        for k in (1, 4, 23):
            a = api.route_forward(x, k, normalize=normalize)
            b = api.route_forward(x0, k, normalize=normalize)
            assert all(torch.equal(u, v) for u, v in zip(a, b))
            dw, v = rand(g, 40, k), rand(g, 40, 23).sign() / 4
            wide = torch.full((40, 29), 7.0, device="cuda")
            d = api.route_backward(dw, x, a[0], a[1], normalize=normalize, dlogits=wide[:, 3:26])
            assert bool((wide[:, :3] == 7).all()) and bool((wide[:, 26:] == 7).all())
            # along v the same experts have to stay chosen: their weights are computed for the same choice
            over = lambda t: (torch.softmax(t.gather(1, a[1].long()), 1) if normalize else torch.softmax(t, 1).gather(1, a[1].long()))      # noqa: E731
            loss = lambda t: (over(t.double()) * dw.double()).sum(1)                                                                       # noqa: E731
            slope = (loss(x0 + h * v) - loss(x0 - h * v)) / (2 * h)
            size = dw.double().abs().amax(1) * 0.25
            assert bool(((d.double() * v).sum(1) - slope).abs().le(size * (h * 0.25) ** 2 * 6 + size * 2.0 ** -18).all())


# ---- moves -------------------------------------------------------------------------------------------------------------

MOVES = [  # tokens, k, cols, rows beyond tokens * k
    (1, 1, 1, 0), (3, 2, 7, 4), (16, 4, 64, 0), (33, 3, 130, 5), (100, 8, 257, 0), (7, 2, 4096, 1), (50, 1, 9000, 0), (5, 32, 40, 0), (300, 2, 1026, 9),
    (2000, 6, 96, 100), (9, 3, 2052, 0), (4, 2, 20001, 0), (64, 5, 514, 0),
]


def places(g, tokens, k, rows):
    """Different rows for all places, some of them empty: -1 or out of range."""
    p = torch.randperm(rows, generator=g, device="cuda")[:tokens * k].view(tokens, k).to(I32)
    gone = torch.rand((tokens, k), generator=g, device="cuda")
    p[gone < 0.1] = -1
    p[gone < 0.06] = rows
    p[gone < 0.04] = 2 ** 31 - 1
    p[gone < 0.02] = -2 ** 31
    return p


def padded(t, extra, shift, fill=NAN):
    big = torch.full((t.shape[0], t.shape[1] + extra + shift), fill, dtype=t.dtype, device="cuda")
    view = big[:, shift:shift + t.shape[1]]
    view.copy_(t)
    return view


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,k,cols,more", MOVES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_moves(tokens, k, cols, more, dtype):
    g = gen(tokens + k + cols)
    rows = tokens * k + more
    p = places(g, tokens, k, rows)
    x, r, y, dy = (rand(g, n, cols, dtype=dtype) for n in (tokens, tokens, rows, tokens))
    w = rand(g, tokens, k)
    some = (p >= 0) & (p < rows)
    w[~some] = NAN                                                           # not read
    at = torch.where(some, p, 0).long()
    weight = w.double().masked_fill(~some, 0)
    # dispatch
    want = torch.full((rows, cols), 3.0, dtype=dtype, device="cuda")
    want[at[some]] = x[:, None].expand(-1, k, -1)[some]
    out = torch.full((rows, cols), 3.0, dtype=dtype, device="cuda")
    assert api.dispatch_forward(x, p, out=out) is out and torch.equal(out, want)
    # combine, with and without weights and residual
    terms = y.double()[at] * weight[..., None]
    sizes = terms.abs().sum(1) + r.double().abs()
    got = api.combine_forward(y, p, w, residual=r)
    within(got, r.double() + terms.sum(1), sizes * (k + 1) * 2.0 ** -24, dtype)
    within(api.combine_forward(y, p, w), terms.sum(1), sizes * (k + 1) * 2.0 ** -24, dtype)
    plain = y.double()[at] * some[..., None]
    within(api.dispatch_backward(y, p), plain.sum(1), plain.abs().sum(1) * k * 2.0 ** -24, dtype)
    within(api.combine_forward(y, p), plain.sum(1), plain.abs().sum(1) * k * 2.0 ** -24, dtype)
    # its gradient
    drows = torch.full((rows, cols), 5.0, dtype=dtype, device="cuda")
    d, dw = api.combine_backward(dy, y, p, w, drows=drows)
    assert d is drows
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[at[some]] = True
    assert bool((drows[~named] == 5).all())
    back = (dy.double()[:, None] * weight[..., None])[some]
    within(drows[at[some]], back, back.abs() * 2.0 ** -24, dtype)
    dots = (dy.double()[:, None] * y.double()[at]).masked_fill(~some[..., None], 0)
    within(dw, dots.sum(2), dots.abs().sum(2) * (cols + 1) * 2.0 ** -24, F32)
    assert torch.equal(dw, api.combine_backward(dy, y, p, w)[1])             # a fixed order
    # strides and bases off 16 bytes
    for extra, shift in ((8, 8), (3, 1), (2, 2)):
        a = api.dispatch_forward(padded(x, extra, shift), p, out=padded(torch.full_like(want, 3.0), 5, 1))
        assert torch.equal(a, want)
        big = torch.full((tokens, cols + 4), 7.0, dtype=dtype, device="cuda")
        b = api.combine_forward(padded(y, extra, shift), p, w, residual=padded(r, 1, 3), out=big[:, 2:2 + cols])
        assert torch.equal(b, got) and bool((big[:, :2] == 7).all()) and bool((big[:, 2 + cols:] == 7).all())
        dd, dw2 = api.combine_backward(padded(dy, extra, shift), padded(y, shift, extra), p, w, drows=padded(torch.full_like(drows, 5.0), extra, shift))
        assert torch.equal(dd, drows)
        within(dw2, dots.sum(2), dots.abs().sum(2) * (cols + 1) * 2.0 ** -24, F32)
    in_place = r.clone()
    assert api.combine_forward(y, p, w, residual=in_place, out=in_place) is in_place and torch.equal(in_place, got)


@pytest.mark.gpu
def test_moves_of_nothing_and_special_values():
    none = torch.empty((0, 8), dtype=BF16, device="cuda")
    empty = torch.empty((0, 2), dtype=I32, device="cuda")
    rows = torch.ones((3, 8), dtype=BF16, device="cuda")
    assert api.dispatch_forward(none, empty).shape == (0, 8) and api.combine_forward(rows, empty).shape == (0, 8)
    assert api.combine_backward(none, rows, empty, torch.empty((0, 2), device="cuda"))[1].shape == (0, 2)
    away = torch.full((4, 2), -1, dtype=I32, device="cuda")                  # tokens that go nowhere, rows there or not
    for r in (rows, none):
        assert not bool(api.dispatch_backward(r, away).any()) and api.dispatch_backward(r, away).shape == (4, 8)
        d, dw = api.combine_backward(rows.new_ones((4, 8)), r, away, torch.full((4, 2), NAN, device="cuda"))
        assert not bool(dw.any())
    y = torch.tensor([[NAN, 1, INF, 1], [1, 1, -INF, 2]], device="cuda")
    p = torch.tensor([[0, 1], [1, -1]], dtype=I32, device="cuda")
    z = api.combine_forward(y, p, torch.ones((2, 2), device="cuda"))
    assert bool(torch.isnan(z[0, 0])) and bool(torch.isnan(z[0, 2])) and z[0, 1] == 2 and z[1].tolist() == [1, 1, -INF, 2]


# ---- products grouped by expert ----------------------------------------------------------------------------------------

GROUPS = [  # rows of each expert, rows before and behind them, in, out
    ([1], 0, 0, 64, 128), ([0], 0, 3, 64, 64), ([2, 0], 0, 0, 1, 1), ([0, 0, 5], 0, 2, 96, 33), ([3, 0, 70, 1], 4, 9, 200, 264),
    ([128, 129, 127], 0, 0, 136, 640), ([257, 0, 1, 300, 64], 0, 50, 512, 520), ([16, 17, 15, 33, 31, 32, 0, 1], 7, 0, 1000, 130),
    ([1000], 0, 0, 72, 2000), ([i % 4 for i in range(70)], 0, 0, 264, 300), ([90, 400, 12], 1, 1, 1021, 515), ([700, 5, 513], 0, 0, 777, 771),
    ([0] * 40 + [3] + [0] * 40 + [260], 0, 0, 128, 256), ([2100, 1800], 0, 100, 256, 768),
    # a few rows: the kernel for those, by row and by expert
    ([0, 0, 2, 0, 1, 0, 0, 3, 0, 0], 1, 2, 520, 130), ([5, 0, 27], 0, 0, 64, 96), ([1, 0, 0, 0, 0, 0, 1], 0, 0, 4096, 520), ([1, 0, 2], 0, 1, 333, 77),
    # several tiles for every block, several of one expert one after the other
    ([5000, 100, 3000], 0, 0, 192, 1536), ([i % 7 for i in range(100)], 0, 0, 512, 512), ([9] * 30, 5, 0, 90, 1000),
]


def ragged(counts, before, behind):
    starts = torch.tensor([before] + counts).cumsum(0)
    return starts.to(I32).cuda(), before + sum(counts) + behind


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(GROUPS)))
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_experts_forward(case, dtype):
    check_forward(case, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(GROUPS)))
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_experts_backward(case, dtype):
    check_backward(case, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [2, 4, 6, 7, 9, 10, 11, 18, 19, 20])
@pytest.mark.parametrize("shape", [1, 2, 3, 4, 5])
def test_experts_on_every_tile_shape(case, shape):
    with api.tuning(test_product_shape=shape):
        check_forward(case, (BF16, F16)[shape % 2])
        check_backward(case, (F16, BF16)[shape % 2])


def check_forward(case, dtype):
    counts, before, behind, k, n = GROUPS[case]
    offsets, rows = ragged(counts, before, behind)
    g, e = gen(case), len(counts)
    x, w = rand(g, rows, k, dtype=dtype), rand(g, e, n, k, scale=k ** -0.5, dtype=dtype)
    activation = api.ACTIVATIONS[case % 4]
    bias = rand(g, e, n, dtype=(BF16, F16, F32)[case % 3])
    x[:before], x[rows - behind:] = NAN, INF                                 # nobody's rows
    fill = lambda: torch.full((rows, n), 7.0, dtype=dtype, device="cuda")    # noqa: E731
    y, pre, plain = fill(), fill(), fill()
    api.experts_forward(x, w, offsets, bias, activation, out=y, pre=pre)
    api.experts_forward(x, w, offsets, out=plain)
    at = before
    for i, c in enumerate(counts):
        z, slack = products(x[at:at + c], w[i])
        within(plain[at:at + c], z, slack, dtype)
        z = z + bias[i].double()
        slack = slack + 2.0 ** -23 * z.abs()
        within(pre[at:at + c], z, slack, dtype)
        want = act64(z, activation)
        within(y[at:at + c], want, slack * STEEPEST[activation] + 2.0 ** -20 * (z.abs() + want.abs()), dtype)
        at += c
    for t in (y, pre, plain):
        assert bool((t[:before] == 7).all()) and bool((t[rows - behind:] == 7).all())


def check_backward(case, dtype):
    counts, before, behind, k, n = GROUPS[case]
    offsets, rows = ragged(counts, before, behind)
    g, e = gen(case + 100), len(counts)
    activation = api.ACTIVATIONS[(case + case // 4) % 4]
    x, w = rand(g, rows, k, dtype=dtype), rand(g, e, n, k, scale=k ** -0.5, dtype=dtype)
    pre, dy = rand(g, rows, n, dtype=dtype), rand(g, rows, n, dtype=dtype)
    for t in (x, pre, dy):
        t[:before], t[rows - behind:] = INF, NAN
    dx = torch.full((rows, k), 7.0, dtype=dtype, device="cuda")
    got = api.experts_backward(dy, x, w, offsets, pre if activation != "none" else None, activation, dx=dx)
    assert got[0] is dx and bool((dx[:before] == 7).all()) and bool((dx[rows - behind:] == 7).all())
    at = before
    for i, c in enumerate(counts):
        here = slice(at, at + c)
        d, xs, wi = dy[here].double(), x[here].double(), w[i].double()
        dz = d * slope64(pre[here].double(), activation)
        off = dz.abs() * HALF_ULP[dtype] * (activation != "none") + d.abs() * 2.0 ** -20 + TINY[dtype]
        within(dx[here], dz @ wi, off @ wi.abs() + (n + 2) * 2.0 ** -23 * (dz.abs() @ wi.abs()), dtype)
        within(got[1][i], dz.T @ xs, off.T @ xs.abs() + (c + 2) * 2.0 ** -23 * (dz.abs().T @ xs.abs()), dtype)
        within(got[2][i], dz.sum(0), (d.abs() * 2.0 ** -20).sum(0) + (c + 2) * 2.0 ** -24 * dz.abs().sum(0), F32)
        at += c
    again = api.experts_backward(dy, x, w, offsets, pre, activation, dx=torch.full_like(dx, 7.0))
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    for need in ((True, False, False), (False, True, False), (False, False, True)):
        part = api.experts_backward(dy, x, w, offsets, pre, activation, need=need, dx=torch.full_like(dx, 7.0))
        assert all((v is None) == (not want) and (v is None or torch.equal(v, f)) for v, want, f in zip(part, need, got))


@pytest.mark.gpu
def test_experts_keep_to_their_rows():
    """Infinities and NaN of one expert's rows or weight stay in its results."""
    counts = [40, 23, 0, 70, 9]
    offsets, rows = ragged(counts, 0, 0)
    g = gen(3)
    for bad in (0, 1, 3, 4):
        x, w, dy = rand(g, rows, 136, dtype=F16), rand(g, 5, 200, 136, scale=0.1, dtype=F16), rand(g, rows, 200, dtype=F16)
        here = slice(int(offsets[bad]), int(offsets[bad + 1]))
        x[here], w[bad], dy[here] = NAN, INF, NAN
        y = api.experts_forward(x, w, offsets)
        dx, dw, db = api.experts_backward(dy, x, w, offsets)
        for t in (y, dx):
            assert not bool(torch.isfinite(t[here]).any())
            t[here] = 0
            assert bool(torch.isfinite(t).all())
        for t in (dw, db):
            assert bool(torch.isnan(t[bad]).all()) and not bool(t[2].any())
            t[bad] = 0
            assert bool(torch.isfinite(t).all())


@pytest.mark.gpu
def test_experts_strides_and_orders():
    counts, k, n = [37, 0, 130, 5], 96, 72
    offsets, rows = ragged(counts, 0, 3)
    g = gen(4)
    x, w, dy = rand(g, rows, k, dtype=BF16), rand(g, 4, n, k, scale=0.1, dtype=BF16), rand(g, rows, n, dtype=BF16)
    bias = rand(g, 4, n)
    used = slice(0, sum(counts))
    want = api.experts_forward(x, w, offsets, bias)[used]
    dx, dw, db = api.experts_backward(dy, x, w, offsets)

    def apart(t, gap, shift, extra):                                         # rows and matrices further apart
        big = torch.full((t.shape[0], t.shape[1] + gap, t.shape[2] + shift + extra), NAN, dtype=t.dtype, device="cuda")
        view = big[:, :t.shape[1], shift:shift + t.shape[2]]
        view.copy_(t)
        return view

    turned = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)        # noqa: E731
    for v in (turned(w), apart(w, 0, 8, 8), apart(w, 3, 8, 0), apart(w, 0, 1, 4), apart(w, 2, 1, 0), apart(w.transpose(1, 2), 1, 3, 2).transpose(1, 2)):
        assert torch.equal(api.experts_forward(x, v, offsets, bias)[used], want)
        got = api.experts_backward(dy, x, v, offsets)
        assert torch.equal(got[0][used], dx[used]) and torch.equal(got[1], dw) and torch.equal(got[2], db)
    for extra, shift in ((8, 8), (3, 1), (0, 2)):
        wide = padded(torch.full((rows, n), 7.0, dtype=BF16, device="cuda"), extra, shift, fill=7.0)
        api.experts_forward(padded(x, extra, shift), w, offsets, padded(bias, extra, shift), out=wide)
        assert torch.equal(wide[used], want) and bool((wide[used.stop:] == 7).all())
        base = wide._base if wide._base is not None else wide
        assert int((base == 7).sum()) >= base.numel() - want.numel()
        grads = apart(torch.zeros_like(dw), 2, shift, extra)
        got = api.experts_backward(padded(dy, extra, shift), padded(x, shift, extra), w, offsets, dx=padded(torch.zeros_like(x), extra, shift), dw=grads)
        assert torch.equal(got[0][used], dx[used]) and torch.equal(grads, dw) and torch.equal(got[2], db)
        assert int(torch.isnan(grads._base).sum()) == grads._base.numel() - dw.numel()      # nothing beside it
    assert torch.equal(api.experts_forward(x, w, offsets, bias[:1].expand(4, n))[:37], want[:37])     # one bias for all


@pytest.mark.gpu
def test_experts_with_offsets_that_are_none():
    """Offsets that decrease or leave the rows: nothing outside the arrays is touched, and the call returns."""
    rows, k, n = 200, 64, 96
    g = gen(5)
    x, w, dy = rand(g, rows, k, dtype=BF16), rand(g, 4, n, k, dtype=BF16), rand(g, rows, n, dtype=BF16)
    for bad in ([0, 50, 20, 100, 200], [-7, 50, 100, 150, 10 ** 9], [2 ** 31 - 1] * 5, [-2 ** 31] * 5, [200, 150, 100, 50, 0], [0, 200, 0, 200, 0]):
        offsets = torch.tensor(bad, dtype=I32, device="cuda")
        room = torch.full((rows + 64, n), 7.0, dtype=BF16, device="cuda")
        api.experts_forward(x, w, offsets, out=room[32:-32])
        for pre, act in ((None, "none"), (dy, "gelu")):
            dx, dw, db = api.experts_backward(dy, x, w, offsets, pre, act)
        torch.cuda.synchronize()
        assert bool((room[:32] == 7).all()) and bool((room[-32:] == 7).all())
    for bad in ([0, 5, 2, 9, 3], [-7, 5, 10, 2, 10 ** 9], [2 ** 31 - 1] * 5, [-2 ** 31] * 5, [8, 6, 4, 2, 0], [0, 8, 0, 8, 0]):     # a few rows
        for experts in (4, 12):                                              # (by expert and by row)
            offsets = torch.tensor(bad + bad[-1:] * (experts - 4), dtype=I32, device="cuda")
            room = torch.full((8 + 64, n), 7.0, dtype=BF16, device="cuda")
            api.experts_forward(x[:8], w.repeat(3, 1, 1)[:experts], offsets, out=room[32:-32])
            torch.cuda.synchronize()
            assert bool((room[:32] == 7).all()) and bool((room[-32:] == 7).all())


@pytest.mark.gpu
def test_experts_no_rows():
    w = torch.ones((3, 40, 24), dtype=BF16, device="cuda")
    none = torch.zeros(4, dtype=I32, device="cuda")
    x, dy = torch.empty((0, 24), dtype=BF16, device="cuda"), torch.empty((0, 40), dtype=BF16, device="cuda")
    assert api.experts_forward(x, w, none).shape == (0, 40)
    for rows in (0, 5):
        dx, dw, db = api.experts_backward(dy.new_ones((rows, 40)), x.new_ones((rows, 24)), w, none)
        assert dx.shape == (rows, 24) and not bool(dw.any()) and not bool(db.any())


@pytest.mark.gpu
@pytest.mark.parametrize("activation", api.ACTIVATIONS)
def test_experts_gradient_against_differences(activation):
    """As for the linear layer: inputs are multiples of 2^-6, so x +- hv is exact; central differences are off by h^2/6 of the
    third derivative along v, and the outputs' rounding, 2^-11 of |y dy|, is divided by h."""
    g = gen(21)
    counts, k, n, h = [9, 0, 14], 16, 40, 2.0 ** -5
    offsets, rows = ragged(counts, 0, 0)
    grid = lambda *s: (torch.randint(-64, 65, s, generator=g, device="cuda") / 64)       # noqa: E731
    x, w, dy = grid(rows, k).to(F16), (grid(3, n, k) / 4).to(F16), grid(rows, n).to(F16)
    if activation == "relu":                                                             # no kink within reach
        x, w = x.abs() + 0.5, w.abs() + 0.0625
    pre = torch.empty((rows, n), dtype=F16, device="cuda")
    y = api.experts_forward(x, w, offsets, activation=activation, pre=pre)
    dx, dw, _ = api.experts_backward(dy, x, w, offsets, pre, activation)
    vx, vw = grid(rows, k).sign().to(F16), (grid(3, n, k).sign() / 4).to(F16)

    def loss(a, b):
        return (api.experts_forward(a, b, offsets, activation=activation).double() * dy.double()).sum()

    third = 4.0 if activation in ("gelu", "silu") else 0.0                               # |f'''| <= 1.6, of |z'|^3
    for d, v, up, down, zp in ((dx, vx, (x + h * vx, w), (x - h * vx, w), w.double().abs().sum(2).amax()),
                               (dw, vw, (x, w + h * vw), (x, w - h * vw), x.double().abs().sum(1).amax() / 4)):
        slope = (loss(*up) - loss(*down)) / (2 * h)
        size = float((y.double() * dy.double()).abs().sum())
        reach = float(dy.double().abs().sum()) * third * float(zp) ** 3 * h * h / 6
        grads = float((d.double() * v.double()).abs().sum())
        assert abs(float((d.double() * v.double()).sum() - slope)) <= size * 2 * 2.0 ** -11 / h + reach + grads * 2 * 2.0 ** -11


@pytest.mark.gpu
@pytest.mark.parametrize("stride", [(1 << 26) + 8, (1 << 26) + 1])
def test_rows_far_apart(stride):
    """40 rows 2^26 elements apart, and five weights 2^30: offsets pass 2^31 elements and 2^32 bytes, on 16-byte boundaries and off
    them."""
    g = gen(30)
    buffer = torch.zeros(40 * stride, dtype=BF16, device="cuda")
    far = lambda t: buffer.as_strided(t.shape, (stride, 1)).copy_(t)                     # noqa: E731
    room = lambda *s: buffer.as_strided(s, (stride, 1)).zero_()                          # noqa: E731
    offsets, rows = ragged([9, 0, 20, 11, 0], 0, 0)
    x, w, dy, pre = rand(g, 40, 72, dtype=BF16), rand(g, 5, 56, 72, dtype=BF16), rand(g, 40, 56, dtype=BF16), rand(g, 40, 56, dtype=BF16)
    few = torch.tensor([0, 3, 3, 8, 8, 8], dtype=I32, device="cuda")
    want, want_few = api.experts_forward(x, w, offsets, activation="gelu"), api.experts_forward(x[:8], w, few)
    assert torch.equal(api.experts_forward(far(x), w, offsets, activation="gelu"), want)
    assert torch.equal(api.experts_forward(far(x)[:8], w, few), want_few)
    assert torch.equal(api.experts_forward(x, w, offsets, activation="gelu", out=room(40, 56)), want)
    assert torch.equal(api.experts_forward(x[:8], w, few, out=room(8, 56)), want_few)
    z = room(40, 56)
    api.experts_forward(x, w, offsets, activation="gelu", pre=z)
    assert torch.equal(z, api.experts_forward(x, w, offsets))
    grads = api.experts_backward(dy, x, w, offsets, pre, "silu")
    for got in (api.experts_backward(far(dy), x, w, offsets, pre, "silu"), api.experts_backward(dy, far(x), w, offsets, pre, "silu"),
                api.experts_backward(dy, x, w, offsets, far(pre), "silu"), api.experts_backward(dy, x, w, offsets, pre, "silu", dx=room(40, 72))):
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
    apart = (1 << 29) + (stride & 15)
    stack = lambda: buffer.as_strided((5, 56, 72), (apart, 72, 1))                       # noqa: E731
    assert 4 * apart + 56 * 72 <= buffer.numel()
    assert torch.equal(api.experts_forward(x, stack().copy_(w), offsets, activation="gelu"), want)
    assert torch.equal(api.experts_forward(x[:8], stack(), few), want_few)
    assert all(torch.equal(a, b) for a, b in zip(api.experts_backward(dy, x, stack(), offsets, pre, "silu"), grads))
    assert torch.equal(api.experts_backward(dy, x, w, offsets, pre, "silu", dw=stack().zero_())[1], grads[1])
    # moves: 20 tokens with two rows each
    p = torch.randperm(40, generator=g, device="cuda").view(20, 2).to(I32)
    t, y, weights = x[:20], rand(g, 40, 72, dtype=BF16), rand(g, 20, 2)
    sent, joined, back = api.dispatch_forward(t, p), api.combine_forward(y, p, weights, residual=t), api.combine_backward(t, y, p, weights)
    assert torch.equal(api.dispatch_forward(far(t), p), sent) and torch.equal(api.dispatch_forward(t, p, out=room(40, 72)), sent)
    assert torch.equal(api.combine_forward(far(y), p, weights, residual=t), joined) and torch.equal(api.combine_forward(y, p, weights, residual=far(t)), joined)
    assert torch.equal(api.combine_forward(y, p, weights, residual=t, out=room(20, 72)), joined)
    near = dict(rtol=1e-5, atol=1e-4)                        # (the order of a sum goes by the alignment)
    for got in (api.combine_backward(far(t), y, p, weights), api.combine_backward(t, far(y), p, weights), api.combine_backward(t, y, p, weights, drows=room(40, 72))):
        assert torch.equal(got[0], back[0]) and torch.allclose(got[1], back[1], **near)
    assert torch.equal(api.dispatch_backward(y, p, dx=room(20, 72)), api.dispatch_backward(y, p))
    logits = rand(g, 40, 24, dtype=BF16)
    routes = api.route_forward(logits, 3, normalize=False)
    assert all(torch.equal(a, b) for a, b in zip(api.route_forward(far(logits), 3, normalize=False), routes))
    dw = rand(g, 40, 3)
    d = api.route_backward(dw, logits, routes[0], routes[1], normalize=False)
    assert torch.equal(api.route_backward(dw, far(logits), routes[0], routes[1], normalize=False), d)
    assert torch.equal(api.route_backward(dw, logits, routes[0], routes[1], normalize=False, dlogits=room(40, 24)), d)


@pytest.mark.gpu
def test_more_than_two_to_the_31_elements():
    """Rows by expert of 140000 x 16000; from the beginning, the middle and the end."""
    g = gen(31)
    counts = [60000, 0, 79990]
    offsets, rows = ragged(counts, 0, 10)
    x, w = rand(g, rows, 64, dtype=BF16), rand(g, 3, 16000, 64, scale=0.1, dtype=BF16)
    y = torch.zeros((rows, 16000), dtype=BF16, device="cuda")
    api.experts_forward(x, w, offsets, activation="relu", out=y)
    for at, e in ((0, 0), (59950, 0), (60000, 2), (134215, 2), (139890, 2)):             # 134218 x 16000 is 2^31
        part = slice(at, at + 50)
        z, slack = products(x[part], w[e])
        within(y[part], act64(z, "relu"), slack, BF16)
    assert not bool(y[139990:].any())
    p = torch.arange(rows, device="cuda", dtype=I32).flip(0).view(-1, 1).contiguous()
    back = api.combine_forward(y, p)
    for at in (0, 5785, 70000, 139950):
        assert torch.equal(back[at:at + 50], y[rows - at - 50:rows - at].flip(0))


# ---- the bound on the gradients -------------------------------------------------------------------------------------------

def norm64(tensors):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


LISTS = [[1], [5, 0, 7], [4096], [100000, 3, 64, 1 << 20], [17] * 40, [1 + i % 50 for i in range(300)], [8193, 8191, 2049], [3] * 1100 + [70000], [3 << 21]]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(LISTS)))
@pytest.mark.parametrize("kind", ["bf16", "f16", "f32", "mixed", "off the blocks"])
def test_clip(case, kind):
    """Up to 64 squares are added in 32 bits (their sums then in 64): 65 2^-24 of the norm's square, half of it of the norm, and
    its rounding; the factor takes three roundings more."""
    g = gen(case)
    types = {"bf16": [BF16], "f16": [F16], "f32": [F32]}.get(kind, [F32, BF16, F16])
    grads = []
    for i, n in enumerate(LISTS[case]):
        shift = i % 9 if kind == "off the blocks" else 0
        grads.append(rand(g, n + shift, scale=0.05, dtype=types[i % len(types)])[shift:])
    total = norm64(grads)
    off = (65 / 2 + 1) * 2.0 ** -24
    keep = [t.clone() for t in grads]
    norm = api.clip_gradients(grads, None)
    assert norm.shape == () and norm.dtype is F32 and abs(float(norm) - total) <= total * off * 1.01
    assert all(torch.equal(a, b) for a, b in zip(grads, keep))
    for bound in (total / 3, total * 2, 0.0):
        factor = min(1.0, bound / (total + 1e-6))
        slack = [t.double().abs() * factor * (off + 4 * 2.0 ** -24) for t in keep]
        out = [torch.full((t.numel() + 16,), 7.0, dtype=t.dtype, device="cuda") for t in keep]
        cut = [o[i % 8:i % 8 + t.numel()] if kind == "off the blocks" else o[8:8 + t.numel()] for i, (o, t) in enumerate(zip(out, keep))]
        again = api.clip_gradients(grads, bound, out=cut)
        assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(grads, keep))
        for o, c, t, s in zip(out, cut, keep, slack):
            within(c, t.double() * factor, s, t.dtype)
            assert int((o == 7).sum()) >= 16                                 # nothing beside it
        work = [t.clone() for t in keep]
        if kind == "off the blocks":
            work = [padded(t[None], 3, 5, fill=3.0)[0] if t.numel() else t for t in work]
        api.clip_gradients(work, bound)
        for a, t, s in zip(work, keep, slack):
            within(a, t.double() * factor, s, t.dtype)


@pytest.mark.gpu
def test_clip_special_values_and_shapes():
    one = lambda *v, dtype=F32: torch.tensor(v, dtype=dtype, device="cuda")              # noqa: E731
    for size in (1e30, 1e-30, 1e-40, 3e38, 1e19, 1e-19):
        t = torch.full((1000,), size, device="cuda")
        t[500:] = 0
        want = norm64([t])
        got = float(api.clip_gradients([t], None))
        assert abs(got - want) <= 2.0 ** -20 * want + 2.0 ** -149 if want < 3.4e38 else got == INF
    mixed = [torch.full((100,), 2.0 ** 100, device="cuda"), torch.full((100,), 2.0 ** -100, device="cuda")]
    assert float(api.clip_gradients(mixed, None)) == 10 * 2.0 ** 100
    zeros = [torch.zeros(100, device="cuda"), torch.zeros(50, dtype=BF16, device="cuda")]
    assert float(api.clip_gradients(zeros, 1.0)) == 0 and not bool(zeros[0].any())
    a = one(1.0, INF, -2.0)
    assert float(api.clip_gradients([a], 1.0)) == INF and a[0] == 0 and bool(torch.isnan(a[1])) and a[2] == 0
    a, b = one(1.0, NAN), one(2.0, dtype=BF16)
    assert bool(torch.isnan(api.clip_gradients([a, b], 1.0))) and bool(torch.isnan(a).all()) and bool(torch.isnan(b).all())
    a = one(3.0, 4.0)
    assert float(api.clip_gradients([a], INF)) == 5 and a.tolist() == [3, 4]
    assert float(api.clip_gradients([], 1.0)) == 0 and float(api.clip_gradients([one()], 1.0)) == 0
    g = gen(2)
    t = rand(g, 30, 50)
    turned, cube = t.clone().T, rand(g, 4, 6, 8, dtype=BF16).permute(2, 0, 1)
    keep = [turned.clone(), cube.clone()]
    norm = float(api.clip_gradients([turned, cube], 1.0))
    for a, b in zip((turned, cube), keep):
        within(a, b.double() * (1.0 / (norm + 1e-6)), b.double().abs() * 2.0 ** -21, a.dtype)
    version = turned._version
    api.clip_gradients([turned], None)
    assert turned._version == version
    api.clip_gradients([turned], 0.5)
    assert turned._version > version


@pytest.mark.gpu
def test_clip_many_elements_in_one_tensor():
    t = torch.ones((1 << 31) + 1000, dtype=BF16, device="cuda")
    assert abs(float(api.clip_gradients([t], 1.0)) - math.sqrt(t.numel())) < 1e-5 * math.sqrt(t.numel())
    want = torch.tensor(1.0 / (math.sqrt(t.numel()) + 1e-6)).bfloat16()
    assert bool((t[:1000] == want).all()) and bool((t[-1000:] == want).all()) and bool((t[(1 << 31) - 500:(1 << 31) + 500] == want).all())


# ---- all of them --------------------------------------------------------------------------------------------------------------

def block(x, wr, w1, w2, b1, k, dy, stream=None):
    """A block of experts forwards and backwards, as a training step runs it."""
    logits = api.linear_forward(x, wr, stream=stream)
    weights, choice, position, offsets = api.route_forward(logits, k, stream=stream)
    rows = api.dispatch_forward(x, position, stream=stream)
    z = torch.zeros((rows.shape[0], w1.shape[1]), dtype=x.dtype, device="cuda")
    u = api.experts_forward(rows, w1, offsets, b1, "gelu", pre=z, stream=stream)
    v = api.experts_forward(u, w2, offsets, stream=stream)
    y = api.combine_forward(v, position, weights, residual=x, stream=stream)
    dv, dweights = api.combine_backward(dy, v, position, weights, stream=stream)
    du, dw2, _ = api.experts_backward(dv, u, w2, offsets, need=(True, True, False), stream=stream)
    drows, dw1, db1 = api.experts_backward(du, rows, w1, offsets, z, "gelu", stream=stream)
    dx = api.dispatch_backward(drows, position, stream=stream)
    dlogits = api.route_backward(dweights, logits, weights, choice, stream=stream)
    dxr, dwr, _ = api.linear_backward(dlogits, x, wr, stream=stream)
    grads = [dw1, dw2, db1, dwr]
    norm = api.clip_gradients(grads, 0.5, stream=stream)
    return [y, dx, dxr, norm, *grads]


def block_inputs(tokens=120, d=72, f=136, experts=6, k=2):
    g = gen(9)
    return (rand(g, tokens, d, dtype=BF16), rand(g, experts, d, scale=d ** -0.5, dtype=BF16), rand(g, experts, f, d, scale=d ** -0.5, dtype=BF16),
            rand(g, experts, d, f, scale=f ** -0.5, dtype=BF16), rand(g, experts, f, scale=0.1), k, rand(g, tokens, d, scale=0.1, dtype=BF16))


@pytest.mark.gpu
def test_block_on_another_stream_and_in_a_graph():
    inputs = block_inputs()
    want = block(*inputs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = block(*inputs, stream=s)
    with torch.cuda.stream(s):
        inside = block(*inputs)
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and all(torch.equal(a, b) for a, b in zip(want, inside))
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    x = inputs[0].clone()
    with torch.cuda.graph(graph):
        out = block(x, *inputs[1:])
    with torch.cuda.graph(other, pool=graph.pool()):
        second = block(inputs[0], *inputs[1:])
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
    x.copy_(inputs[0].flip(0))                                               # other data: other offsets
    graph.replay()
    changed = block(x, *inputs[1:])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(changed, out)) and not torch.equal(out[0], want[0])
    other.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, second))


@pytest.mark.gpu
def test_block_gradients_against_autograd():
    """bfloat16 tensors between the operators: sqrt(8) of them, 2^-9 each on average, four times that allowed."""
    x, wr, w1, w2, b1, k, dy = block_inputs()
    got = block(x, wr, w1, w2, b1, k, dy)
    leaves = [t.float().requires_grad_() for t in (x, wr, w1, w2, b1)]
    X, R, A, B, C = leaves
    logits = X @ R.T
    value, index = api.linear_forward(x, wr).float().topk(k, 1)              # the choice of the rounded logits
    p = torch.softmax(logits.gather(1, index), 1)
    y = X
    for j in range(k):
        e = index[:, j]
        u = torch.einsum("td,tfd->tf", X, A[e]) + C[e]
        u = u * 0.5 * torch.special.erfc(-u / 2 ** 0.5)
        y = y + p[:, j:j + 1] * torch.einsum("tf,tdf->td", u, B[e])
    y.backward(dy.float())
    norm = math.sqrt(sum(float((t.grad ** 2).sum()) for t in (A, B, C, R)))
    assert abs(float(got[3]) - norm) < 0.022 * norm
    factor = min(1.0, 0.5 / norm)
    wants = [y.detach(), X.grad - dy.float(), *[t.grad * factor for t in (A, B, C, R)]]
    gots = [got[0], got[1].float() + got[2].float(), *got[4:]]
    for i, (a, b) in enumerate(zip(gots, wants)):
        assert float((a.float() - b).norm() / b.norm()) < 0.022, i


@pytest.mark.gpu
def test_scratch_is_enough_and_nothing_else_is_written():
    g = gen(10)
    offsets, rows = ragged([30, 0, 41], 0, 2)
    x, w, dy, pre = (rand(g, *s, dtype=BF16) for s in ((rows, 131), (3, 65, 131), (rows, 65), (rows, 65)))
    logits = rand(g, 3000, 40)
    grads = [rand(g, 5000), rand(g, 77, dtype=F16)]
    own = api._operators()
    real, sizes = own.strided, []

    def empty(*a, **kw):                                                     # what the binding allocates for itself
        if kw.get("dtype") == torch.uint8:
            sizes.append(a[0][0])
        return real(*a, **kw)

    calls = (lambda s: api.experts_forward(x, w, offsets, scratch=s), lambda s: api.experts_backward(dy, x, w, offsets, pre, "silu", scratch=s),
             lambda s: api.route_forward(logits, 3, scratch=s), lambda s: api.clip_gradients(grads, 1.0, scratch=s))
    try:
        own.strided = empty
        for call in calls:
            call(None)
    finally:
        own.strided = real
    assert len(sizes) == 4
    for call, need in zip(calls, sizes):
        big = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        call(big[1024:1024 + need])
        torch.cuda.synchronize()
        assert bool((big[:1024] == 0xA5).all()) and bool((big[1024 + need:] == 0xA5).all())
        for bad, status in ((big[1024:1024 + need // 256 * 256 - 256], 5), (big[1025:1025 + need], 7)):
            with pytest.raises(api.RedistError) as e:
                call(bad)
            assert e.value.status == status


@pytest.mark.gpu
def test_a_wait_that_runs_out_is_counted_and_returns():
    offsets, rows = ragged([300, 40, 700], 0, 0)
    g = gen(12)
    x, w, dy = rand(g, rows, 640, dtype=BF16), rand(g, 3, 600, 640, dtype=BF16), rand(g, rows, 600, dtype=BF16)
    want = api.experts_forward(x, w, offsets)
    before = api.redist_product_timeouts()
    with api.tuning(wait_polls=64, test_extra_tx=16):
        for call in (lambda: api.experts_forward(x, w, offsets), lambda: api.experts_backward(dy, x, w, offsets)):
            call()
            after = api.redist_product_timeouts()
            assert after > before
            before = after
    assert torch.equal(api.experts_forward(x, w, offsets), want) and api.redist_product_timeouts() == before


# ---- refusals (no GPU) ---------------------------------------------------------------------------------------------------------

ROUTE = dict(tokens=8, experts=16, chosen=2, type=2, normalize=1, logits=(0x10000, 16, 1), weights=0x20000, choice=0x30000, position=0x40000, offsets=0x50000)
MOVE = dict(tokens=8, rows=16, cols=32, type=0, chosen=2, token=(0x10000, 32, 1), row=(0x20000, 32, 1), residual=(None, 0, 0), drow=(0x30000, 32, 1),
            position=0x40000, weights=0x50000, dweights=0x60000)
EXPERTS = dict(rows=8, in_features=16, out_features=24, experts=3, type=0, bias_type=0, activation=0, x=(0x10000, 16, 1), w=(0x20000, 16, 1),
               out=(0x30000, 24, 1), pre=(None, 0, 0), w_stride=384, bias_stride=24, bias=None, offsets=0x40000)
GRADS = dict(dy=(0x50000, 24, 1), dx=(0x60000, 16, 1), dw=(0x70000, 16, 1), dw_stride=384, dbias=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), 1), (dict(experts=0), 1), (dict(chosen=0), 1), (dict(chosen=17), 1), (dict(type=3), 1), (dict(normalize=2), 1), (dict(experts=1025), 10),
    (dict(experts=64, chosen=33, logits=(0x10000, 64, 1)), 10), (dict(tokens=1 << 30), 10), (dict(logits=(None, 16, 1)), 1), (dict(logits=(0x10000, 15, 1)), 1),
    (dict(logits=(0x10000, 1, 8)), 1), (dict(logits=(0x10002, 16, 1)), 7), (dict(weights=None), 1), (dict(choice=None), 1), (dict(position=None), 1),
    (dict(offsets=None), 1), (dict(offsets=0x50002), 7), (dict(choice=0x20000), 6), (dict(weights=0x10010), 6), (dict(offsets=0x40010), 6),
    (dict(tokens=2000, weights=0x40000, choice=0x50000, position=0x60000, offsets=0x70000), 5),
])
def test_route_refusals(change, status):
    assert api.load().redist_route_forward(api._Route(*{**ROUTE, **change}.values()), None, 0, None) == status


@pytest.mark.parametrize("change,dweights,dlogits,status", [
    (dict(), None, (0x70000, 16, 1), 1), (dict(), 0x60002, (0x70000, 16, 1), 7), (dict(), 0x60000, (None, 16, 1), 1), (dict(), 0x60000, (0x70000, 15, 1), 1),
    (dict(weights=None), 0x60000, (0x70000, 16, 1), 1), (dict(choice=None), 0x60000, (0x70000, 16, 1), 1), (dict(), 0x60000, (0x60010, 16, 1), 6),
    (dict(normalize=0), 0x60000, (0x10000, 16, 1), 6), (dict(normalize=0, logits=(None, 16, 1)), 0x60000, (0x70000, 16, 1), 1),
])
def test_route_backward_refusals(change, dweights, dlogits, status):
    assert api.load().redist_route_backward(api._Route(*{**ROUTE, **change}.values()), dweights, api._Matrix(*dlogits), None) == status


@pytest.mark.parametrize("name", ["dispatch_forward", "dispatch_backward", "combine_forward", "combine_backward"])
@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), 1), (dict(rows=-1), 1), (dict(cols=0), 1), (dict(chosen=0), 1), (dict(chosen=33), 10), (dict(type=3), 1), (dict(cols=(1 << 25) + 1), 10),
    (dict(position=None), 1), (dict(position=0x40002), 7), (dict(token=(None, 32, 1)), 1), (dict(row=(None, 32, 1)), 1), (dict(row=(0x20000, 31, 1)), 1),
    (dict(token=(0x10001, 32, 1)), 7), (dict(row=(0x10010, 32, 1), drow=(0x10010, 32, 1)), 6), (dict(tokens=1 << 31), 10),
])
def test_move_refusals(name, change, status):
    assert getattr(api.load(), "redist_" + name)(api._Move(*{**MOVE, **change}.values()), None) == status


@pytest.mark.parametrize("name", ["dispatch_forward", "dispatch_backward", "combine_forward", "combine_backward"])
def test_widest_moves(name):
    """The last number of columns that is taken, and the next (neither call has a token to move)."""
    def call(cols):
        return getattr(api.load(), "redist_" + name)(api._Move(*{**MOVE, "cols": cols, "token": (None, cols, 1)}.values()), None)
    assert call(65535 * 512) == 1 and call(65535 * 512 + 1) == 10


@pytest.mark.gpu
def test_widest_moves_by_single_elements():
    cols = 65535 * 512
    g = gen(11)
    x = rand(g, 1, cols + 1)[:, 1:]                           # off the blocks of 8 and 16 bytes
    position, weights = torch.zeros((1, 1), dtype=I32, device="cuda"), torch.full((1, 1), 0.5, device="cuda")
    rows = torch.zeros((1, cols + 1), device="cuda")[:, 1:]
    assert torch.equal(api.dispatch_forward(x, position, out=rows), x)
    assert torch.equal(api.combine_forward(rows, position, weights), x * 0.5)
    ones = torch.ones_like(x)
    drows, dweights = api.combine_backward(ones, rows, position, weights, drows=torch.empty((1, cols + 1), device="cuda")[:, 1:])
    assert bool((drows == 0.5).all())
    total = float(x.double().sum())
    # a thread adds some 131072 values one after the other, then 256 such sums meet
    assert abs(float(dweights) - total) <= (cols / 256 + 16) * 2.0 ** -24 * float(x.double().abs().sum())


@pytest.mark.parametrize("name,change,status", [
    ("combine_forward", dict(residual=(0x10010, 32, 1)), 6), ("combine_forward", dict(residual=(0x70000, 31, 1)), 1), ("combine_forward", dict(weights=0x50002), 7),
    ("combine_forward", dict(weights=0x10000), 6), ("combine_backward", dict(weights=None), 1), ("combine_backward", dict(dweights=None), 1),
    ("combine_backward", dict(dweights=0x30000), 6), ("combine_backward", dict(dweights=0x50000), 6), ("combine_backward", dict(drow=(0x20000, 32, 1)), 6),
    ("combine_backward", dict(drow=(None, 32, 1)), 1), ("dispatch_forward", dict(position=0x20000), 6), ("dispatch_backward", dict(position=0x10000), 6),
])
def test_more_move_refusals(name, change, status):
    assert getattr(api.load(), "redist_" + name)(api._Move(*{**MOVE, **change}.values()), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), 1), (dict(in_features=0), 1), (dict(out_features=0), 1), (dict(experts=0), 1), (dict(experts=65536), 10), (dict(type=2), 1),
    (dict(activation=4), 1), (dict(offsets=None), 1), (dict(offsets=0x40002), 7), (dict(x=(None, 16, 1)), 1), (dict(x=(0x10000, 1, 8)), 1),
    (dict(w=(None, 16, 1)), 1), (dict(w_stride=383), 1), (dict(w_stride=0), 1), (dict(w_stride=-384), 1), (dict(w=(0x20001, 16, 1)), 7),
    (dict(out=(0x30000, 23, 1)), 1), (dict(out=(0x10010, 24, 1)), 6), (dict(pre=(0x30010, 24, 1)), 6), (dict(out=(0x20800, 24, 1)), 6),
    (dict(bias=0x50001), 7), (dict(bias=0x50000, bias_type=3), 1), (dict(bias=0x50000, bias_stride=-1), 1), (dict(bias=0x30010), 6),
    (dict(offsets=0x30010), 6), (dict(rows=1 << 31), 10),
    # (a few rows need no scratch)
    (dict(rows=40, x=(0x10002, 16, 1)), 5), (dict(rows=40, w=(0x20002, 16, 1)), 5), (dict(rows=40, w_stride=388), 5),
])
def test_experts_refusals(change, status):
    assert api.load().redist_experts_forward(api._Experts(*{**EXPERTS, **change}.values()), None, 0, None) == status


@pytest.mark.parametrize("change,grads,status", [
    (dict(), dict(dy=(None, 24, 1)), 1), (dict(activation=1), dict(), 1), (dict(), dict(dx=(0x60000, 15, 1)), 1), (dict(), dict(dw=(0x70000, 15, 1)), 1),
    (dict(), dict(dw=(0x70000, 1, 24)), 1), (dict(), dict(dw_stride=383), 1), (dict(), dict(dx=(0x10000, 16, 1)), 6), (dict(), dict(dw=(0x60000, 16, 1)), 6),
    (dict(), dict(dbias=0x70002), 7), (dict(), dict(dbias=0x70000), 6), (dict(), dict(), 5), (dict(x=(None, 0, 0)), dict(), 1), (dict(w=(None, 0, 0)), dict(), 1),
    (dict(), dict(dw=(0x20000, 16, 1)), 6), (dict(rows=0), dict(dbias=0x70000), 6),
])
def test_experts_backward_refusals(change, grads, status):
    op = api._Experts(*{**EXPERTS, **change, "out": (None, 0, 0)}.values())
    assert api.load().redist_experts_backward(op, api._ExpertsGrads(*{**GRADS, **grads}.values()), None, 0, None) == status


@pytest.mark.parametrize("entries,change,status", [
    ([(0x10000, None, -1, 0, 0)], {}, 1), ([(None, None, 5, 0, 0)], {}, 1), ([(0x10000, None, 5, 3, 0)], {}, 1), ([(0x10000, None, 5, 0, 1)], {}, 1),
    ([(0x10001, None, 5, 0, 0)], {}, 7), ([(0x10000, 0x20002, 5, 2, 0)], {}, 7), ([(0x10000, None, 5, 0, 0)], dict(eps=-1.0), 1),
    ([(0x10000, None, 5, 0, 0)], dict(eps=NAN), 1), ([(0x10000, None, 5, 0, 0)], dict(max_norm=NAN), 1), ([(0x10000, None, 5, 0, 0)], dict(norm=0x40002), 7),
    ([(0x10000, None, (1 << 40) + 1, 0, 0)], {}, 10), ([(0x10000, None, 5, 0, 0)], {}, 5),
    ([(0x10000, None, 100, 2, 0), (0x10000, None, 100, 2, 0)], dict(scratch=0x900000), 6), ([(0x10000, None, 100, 2, 0), (0x10010, 0x50000, 10, 2, 0)], dict(scratch=0x900000), 6),
    ([(0x10000, 0x10010, 100, 2, 0)], dict(scratch=0x900000), 6), ([(0x10000, None, 100, 2, 0)], dict(scratch=0x900000, norm=0x10010), 6),
    ([(0x10000, None, 100, 2, 0)], dict(scratch=0x10000), 6), ([(0x10000, 0x30000, 100, 2, 0), (0x20000, 0x30010, 100, 2, 0)], dict(scratch=0x900000), 6),
    ([(0x10000, None, 5, 0, 0)], dict(scratch=0x900001), 7),
])
def test_clip_refusals(entries, change, status):
    change = dict(change)
    scratch = change.pop("scratch", None)
    table = (api._Tensor * len(entries))(*[api._Tensor(*e) for e in entries])
    f = dict(tensors=table, count=len(entries), max_norm=1.0, eps=1e-6, norm=0x800000)
    f.update(change)
    assert api.load().redist_clip(api._Clip(*f.values()), scratch, 1 << 16 if scratch else 0, None) == status


def test_null_arguments_are_refused():
    lib = api.load()
    assert lib.redist_route_forward(None, None, 0, None) == 1 and lib.redist_route_backward(None, None, None, None) == 1
    for name in ("dispatch_forward", "dispatch_backward", "combine_forward", "combine_backward"):
        assert getattr(lib, "redist_" + name)(None, None) == 1
    assert lib.redist_experts_forward(None, None, 0, None) == 1 and lib.redist_experts_backward(None, None, None, 0, None) == 1
    assert lib.redist_clip(None, None, 0, None) == 1 and lib.redist_clip_scratch_bytes(None) == 0
    assert lib.redist_route_scratch_bytes(None) == 0 and lib.redist_experts_scratch_bytes(None, None) == 0


def test_structures_are_those_of_the_packed_blocks():
    for cls, pack, n in ((api._Route, api._pack_route, 12), (api._Move, api._pack_move, 20), (api._Experts, api._pack_experts, 23),
                         (api._ExpertsGrads, api._pack_experts_grads, 11), (api._Clip, api._pack_clip, 5)):
        assert len(pack(*range(n))) == ctypes.sizeof(cls)
    assert ctypes.sizeof(api._Tensor) == 4 * 8 and api._Tensor.type.offset == 24        # four words per tensor


def test_the_binding_refuses_before_the_foreign_call():
    x, p = torch.zeros((4, 8), dtype=BF16), torch.zeros((4, 2), dtype=I32)
    w, o, f = torch.zeros((3, 6, 8), dtype=BF16), torch.zeros(4, dtype=I32), torch.zeros((4, 2))
    for call in (lambda: api.route_forward(x, 2), lambda: api.route_forward(x, 0), lambda: api.route_forward(x, 9), lambda: api.route_forward(x[0], 1),
                 lambda: api.route_backward(f, x, f, p), lambda: api.dispatch_forward(x, p), lambda: api.dispatch_backward(x, p),
                 lambda: api.combine_forward(x, p), lambda: api.combine_backward(x, x, p, f), lambda: api.experts_forward(x, w, o),
                 lambda: api.experts_forward(x, w[0], o), lambda: api.experts_backward(torch.zeros((4, 6), dtype=BF16), x, w, o),
                 lambda: api.clip_gradients([x], 1.0), lambda: api.clip_gradients([x], -1.0), lambda: api.clip_gradients([x], NAN),
                 lambda: api.clip_gradients([x], 1.0, out=[])):
        with pytest.raises(api.RedistError) as e:
            call()                                                           # host tensors, vectors, wrong options
        assert e.value.status == 1


@pytest.mark.gpu
def test_the_binding_refuses_mismatched_tensors():
    c = lambda *s, dtype=BF16: torch.zeros(s, dtype=dtype, device="cuda")                # noqa: E731
    x, p, w, o, f = c(4, 8), c(4, 2, dtype=I32), c(3, 6, 8), c(4, dtype=I32), c(4, 2, dtype=F32)
    lg = c(4, 5, dtype=F32)
    for call in (lambda: api.route_forward(c(4, 5, dtype=torch.float64), 2), lambda: api.route_backward(f, lg, f, p.long()),
                 lambda: api.route_backward(f[:3], lg, f, p), lambda: api.route_backward(f, lg, f, p, dlogits=c(4, 5)),
                 lambda: api.dispatch_forward(x, p.long()), lambda: api.dispatch_forward(x, p[:3]), lambda: api.dispatch_forward(x, p, out=c(8, 7)),
                 lambda: api.dispatch_forward(x, p, out=c(8, 8, dtype=F16)), lambda: api.combine_forward(c(8, 8), p, weights=f.bfloat16()),
                 lambda: api.combine_forward(c(8, 8), p, residual=c(5, 8)), lambda: api.combine_backward(x, c(8, 7), p, f),
                 lambda: api.combine_backward(x, c(8, 8), p, None), lambda: api.experts_forward(x, w, o[:3]), lambda: api.experts_forward(x, w, o.long()),
                 lambda: api.experts_forward(x, w.half(), o), lambda: api.experts_forward(x, w, o, bias=c(3, 5)), lambda: api.experts_forward(x, w, o, bias=c(6)),
                 lambda: api.experts_forward(x, w, o, pre=c(4, 5)), lambda: api.experts_forward(x, w[:, :, ::2], o), lambda: api.experts_forward(x.T, w, o),
                 lambda: api.experts_forward(x, w[:1].expand(3, 6, 8), o), lambda: api.experts_backward(c(4, 6), x, w, o, activation="gelu"),
                 lambda: api.experts_backward(c(4, 6), x, w, o, dw=c(3, 8, 6)), lambda: api.experts_backward(c(4, 5), x, w, o),
                 lambda: api.clip_gradients([x[:, ::2]], 1.0), lambda: api.clip_gradients([x.double()], 1.0), lambda: api.clip_gradients([x, x], 1.0),
                 lambda: api.clip_gradients([x], 1.0, out=[c(8, 4)]), lambda: api.clip_gradients([x], 1.0, out=[x.float()]),
                 lambda: api.clip_gradients([x, x.cpu()], 1.0)):
        with pytest.raises(api.RedistError):
            call()
    torch.cuda.synchronize()
