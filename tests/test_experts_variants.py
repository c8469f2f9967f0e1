"""Variants of the products grouped by expert that take particular sizes to reach -- a few rows of one expert, rows in turns over
blocks that share a sum, weights off 16-byte boundaries of experts most of which are idle, very many experts -- and what lies beside
the arrays that the operators of a block of experts and clipping write.

Tolerances as in the other tests of these operators.
"""
import pytest

from paper_2112_01075_b200 import api
from test_operators import BF16, F16, F32, HALF_ULP, STEEPEST, TINY, act64, gen, rand, slope64, within

torch = pytest.importorskip("torch")

I32 = torch.int32
MARK = 7.0


@pytest.fixture(autouse=True)
def no_wait_runs_out(request):
    before = api.redist_product_timeouts() if "gpu" in request.keywords else 0
    yield
    assert "gpu" not in request.keywords or api.redist_product_timeouts() == before


class Guarded:
    """A tensor of MARK within a larger one of MARK: nothing but what is asked for may have changed around it."""

    def __init__(self, *shape, dtype=BF16, shift=0, extra=0, apart=0):
        lead, cols = shape[:-1], shape[-1]
        if len(lead) == 2:
            lead = (lead[0], lead[1] + apart)
        self.base = torch.full((64 + int(torch.tensor(lead).prod()) * (cols + extra) + 64 + shift,), MARK, dtype=dtype, device="cuda")
        inner = self.base[64 + shift:64 + shift + int(torch.tensor(lead).prod()) * (cols + extra)].view(*lead, cols + extra)
        self.t = inner[:, :shape[1], :cols] if len(shape) == 3 else inner[:, :cols]

    def intact(self, written=None):
        """Beside the tensor, and in its rows that `written` (a mask) does not name."""
        mask = torch.zeros(self.base.shape, dtype=torch.bool, device="cuda")
        inside = torch.as_strided(mask, self.t.shape, self.t.stride(), self.t.storage_offset())
        inside[:] = True if written is None else written[:, None]
        return bool((self.base[~mask] == MARK).all())


def ranges(counts, before, behind):
    offsets = torch.tensor([before] + list(counts)).cumsum(0)
    rows = before + sum(counts) + behind
    owner = torch.full((rows,), -1, dtype=torch.int64)
    owner[before:rows - behind] = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts))
    return offsets.to(I32).cuda(), rows, owner.cuda()


def check(counts, before, behind, k, n, dtype, activation, w_shift=0, extra=0, shift=0, backward=True):
    offsets, rows, owner = ranges(counts, before, behind)
    e, g = len(counts), gen(sum(counts) + len(counts) + k + n)
    used = owner >= 0
    x = rand(g, rows, k, dtype=dtype)
    flat = torch.empty(e * n * k + 64, dtype=dtype, device="cuda")
    w = flat[w_shift:w_shift + e * n * k].view(e, n, k)
    w.copy_(rand(g, e, n, k, scale=k ** -0.5, dtype=dtype))
    bias = rand(g, e, n)
    x[~used] = float("nan")
    y, z = (Guarded(rows, n, dtype=dtype, shift=shift, extra=extra) for _ in range(2))
    api.experts_forward(x, w, offsets, bias, activation, out=y.t, pre=z.t)
    assert y.intact(used) and z.intact(used)
    busy = [(i, (owner == i).nonzero().flatten()) for i, c in enumerate(counts) if c]
    for i, at in busy:
        a, b = x[at].double(), w[i].double()
        want = a @ b.T + bias[i].double()
        slack = (k + 2) * 2.0 ** -23 * (a.abs() @ b.abs().T) + 2.0 ** -23 * want.abs()
        within(z.t[at], want, slack, dtype)
        out = act64(want, activation)
        within(y.t[at], out, slack * STEEPEST[activation] + 2.0 ** -20 * (want.abs() + out.abs()), dtype)
    if not backward:
        return
    pre, dy = rand(g, rows, n, dtype=dtype), rand(g, rows, n, dtype=dtype)
    pre[~used], dy[~used] = float("inf"), float("nan")
    dx, dw, db = Guarded(rows, k, dtype=dtype, shift=shift, extra=extra), Guarded(e, n, k, dtype=dtype, shift=shift, extra=extra, apart=2), Guarded(e, n, dtype=F32)
    db.t.fill_(float("nan"))
    api.experts_backward(dy, x, w, offsets, pre, activation, dx=dx.t, dw=dw.t, dbias=db.t)
    assert dx.intact(used) and dw.intact() and db.intact()
    idle = torch.tensor([c == 0 for c in counts], device="cuda")
    assert not bool(dw.t[idle].any()) and not bool(db.t[idle].any())
    for i, at in busy:
        d, xs, wi = dy[at].double(), x[at].double(), w[i].double()
        dz = d * slope64(pre[at].double(), activation)
        off = dz.abs() * HALF_ULP[dtype] * (activation != "none") + d.abs() * 2.0 ** -20 + TINY[dtype]
        within(dx.t[at], dz @ wi, off @ wi.abs() + (n + 2) * 2.0 ** -23 * (dz.abs() @ wi.abs()), dtype)
        within(dw.t[i], dz.T @ xs, off.T @ xs.abs() + (len(at) + 2) * 2.0 ** -23 * (dz.abs().T @ xs.abs()), dtype)
        within(db.t[i], dz.sum(0), (d.abs() * 2.0 ** -20).sum(0) + (len(at) + 2) * 2.0 ** -24 * dz.abs().sum(0), F32)


# A few rows: one expert with 9 to 16 (two tiles of eight), with 17 to 32 (four), and several experts whose rows come in turns of eight
# over a cluster of blocks; on 32-byte boundaries, on 16-byte ones (by size, or where the weight begins) and off them.
FEW = [  # rows of each expert, before, behind, in, out, elements between a 32-byte boundary and the weight
    ([9], 0, 0, 512, 130, 0), ([16], 0, 0, 1024, 96, 0), ([13], 2, 1, 512, 70, 0), ([12], 0, 0, 520, 64, 0), ([16], 0, 0, 1024, 100, 8), ([11], 1, 2, 264, 33, 0),
    ([10], 0, 0, 4097, 100, 0), ([15], 0, 1, 5001, 256, 0), ([9], 3, 0, 4099, 17, 1),
    ([32], 0, 0, 512, 96, 0), ([17], 0, 0, 520, 96, 0), ([14, 17], 0, 0, 520, 200, 0), ([0, 30], 1, 1, 1024, 64, 8), ([21, 0, 9], 0, 2, 264, 120, 0),
    ([32], 0, 0, 4097, 96, 0), ([18, 13], 0, 1, 4099, 130, 0), ([0, 25], 2, 0, 6001, 40, 3),
    ([20, 0, 9, 3], 0, 0, 8192, 64, 0), ([9, 23, 0, 0], 0, 0, 8200, 50, 0), ([1, 17, 0, 11], 2, 1, 8193, 77, 0), ([0, 0, 29, 0, 3], 0, 0, 4096, 128, 8),
    ([0] * 20 + [26] + [0] * 20 + [2, 0], 1, 3, 4096, 32, 0), ([0] * 9 + [12, 0, 19] + [0] * 30, 0, 1, 5003, 60, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(FEW)))
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_few_rows(case, dtype):
    counts, before, behind, k, n, shift = FEW[case]
    check(counts, before, behind, k, n, dtype, api.ACTIVATIONS[case % 4], w_shift=shift, backward=False)


# Weights off 16-byte boundaries: only those of experts that have rows are laid out, found by the rows where these are fewer than
# the experts.  (Fewer than 33 rows here are too much work for the kernel for a few rows.)
IDLE = [  # rows of each expert, before, behind, in, out
    ([0] * 5 + [1, 0, 2, 0, 0, 3] + [0] * 40 + [4] + [0] * 50 + [1, 1, 0, 1] + [0] * 6, 1, 0, 149, 650),
    ([1] * 14 + [0] * 98, 0, 0, 149, 650), ([0] * 98 + [1] * 14, 0, 0, 149, 650), ([0] * 30 + [14] + [0] * 81, 0, 0, 149, 650),
    ([0, 3] * 3 + [0] * 50 + [5, 6] + [0] * 12, 0, 0, 333, 515), ([0] * 8 + [7] + [0] * 52 + [9] + [0] * 8, 2, 2, 333, 515),
    ([2, 0] * 20 + [0] * 30, 3, 5, 77, 90), ([0] * 69 + [40], 0, 7, 77, 201), ([40] + [0] * 69, 4, 0, 201, 77), ([0] * 33 + [17, 0, 0, 18] + [0] * 33, 0, 0, 1021, 130),
    ([0, 0, 1] * 40, 0, 0, 91, 270),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(IDLE)))
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("extra,shift", [(0, 0), (3, 1)])
def test_idle_experts_with_weights_off_boundaries(case, dtype, extra, shift):
    counts, before, behind, k, n = IDLE[case]
    check(counts, before, behind, k, n, dtype, api.ACTIVATIONS[case % 4], extra=extra, shift=shift)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("counts,before,behind,k,n", [
    ([i % 3 for i in range(600)], 0, 0, 40, 72), ([i % 3 for i in range(513)], 3, 2, 41, 77), ([20 + i % 2 for i in range(600)], 5, 0, 40, 264),
    ([0] * 300 + [700, 0, 0, 900] + [0] * 300, 0, 9, 96, 520),
])
def test_more_experts_than_are_held_in_shared_memory(counts, before, behind, k, n, dtype):
    check(counts, before, behind, k, n, dtype, "silu")


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[0] * 1000 + [3, 0, 17] + [0] * 3100 + [20] + [0] * 100, [i % 100 == 7 for i in range(4200)]])
def test_thousands_of_experts_with_weights_off_boundaries(counts):
    check([int(c) for c in counts], 1, 2, 9, 5, BF16, "gelu")


# ---- what lies beside the arrays ----------------------------------------------------------------------------------------------

@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("tokens,k,cols", [(3, 2, 7), (16, 4, 64), (33, 3, 130), (7, 2, 4097), (100, 8, 257), (50, 1, 9001), (9, 5, 2052), (300, 2, 31)])
@pytest.mark.parametrize("extra,shift", [(0, 0), (8, 8), (3, 1), (2, 2), (5, 3), (1, 7)])
def test_moves_write_their_rows_and_nothing_beside_them(tokens, k, cols, extra, shift, dtype):
    g = gen(tokens + cols)
    rows = tokens * k + 5
    p = torch.randperm(rows, generator=g, device="cuda")[:tokens * k].view(tokens, k).to(I32)
    p[torch.rand((tokens, k), generator=g, device="cuda") < 0.1] = -1
    named = torch.zeros(rows, dtype=torch.bool, device="cuda")
    named[p[p >= 0].long()] = True
    x, y, w = rand(g, tokens, cols, dtype=dtype), rand(g, rows, cols, dtype=dtype), rand(g, tokens, k)
    place = dict(dtype=dtype, shift=shift, extra=extra)
    sent, back = Guarded(rows, cols, **place), Guarded(rows, cols, **place)
    api.dispatch_forward(x, p, out=sent.t)
    _, dw = api.combine_backward(x, y, p, w, drows=back.t)
    joined, dx = Guarded(tokens, cols, **place), Guarded(tokens, cols, **place)
    api.combine_forward(y, p, w, residual=x, out=joined.t)
    api.dispatch_backward(y, p, dx=dx.t)
    assert sent.intact(named) and back.intact(named) and joined.intact() and dx.intact()
    at, some = p.clamp(min=0).long(), p >= 0
    assert torch.equal(sent.t[p[some].long()], x[:, None].expand(-1, k, -1)[some])
    within(dx.t, (y.double()[at] * some[..., None]).sum(1), (y.double()[at].abs() * some[..., None]).sum(1) * k * 2.0 ** -24, dtype)
    in_place = Guarded(tokens, cols, **place)
    in_place.t.copy_(x)
    api.combine_forward(y, p, w, residual=in_place.t, out=in_place.t)
    assert in_place.intact() and torch.equal(in_place.t, joined.t)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 63, 1000, 16385, 32768 + 5, 100003])
def test_clipping_writes_its_tensors_and_nothing_beside_them(n, dtype):
    g = gen(n)
    for shift in range(9):
        place = Guarded(1, n, dtype=dtype, shift=shift)
        values = rand(g, n, dtype=dtype)
        place.t.copy_(values[None])
        apart = Guarded(1, n, dtype=dtype, shift=8 - shift)
        norm = float(api.clip_gradients([place.t[0]], 1e-3, out=[apart.t[0]]))
        assert torch.equal(place.t[0], values) and place.intact() and apart.intact()
        api.clip_gradients([place.t[0]], 1e-3)
        assert place.intact() and torch.equal(place.t, apart.t)
        within(place.t[0], values.double() * (1e-3 / (norm + 1e-6)), values.double().abs() * 1e-3 / norm * 2.0 ** -21, dtype)


@pytest.mark.gpu
def test_offsets_that_are_none_reach_nothing_beside_the_gradients():
    """As documented: what such offsets give is not defined, but nothing outside the arrays and the scratch is written."""
    g = gen(5)
    for rows, e, k, n in ((200, 4, 64, 96), (200, 4, 63, 97), (8, 12, 64, 96), (40, 70, 77, 90)):
        x, w = rand(g, rows, k, dtype=BF16), rand(g, e, n, k, dtype=BF16)
        dy, pre = rand(g, rows, n, dtype=BF16), rand(g, rows, n, dtype=BF16)
        some = [0, rows // 4, rows // 10, rows // 2, rows]
        for bad in (some, [-7, 3, 5, 2, 10 ** 9], [2 ** 31 - 1] * 5, [-2 ** 31] * 5, some[::-1], [0, rows, 0, rows, 0]):
            offsets = torch.tensor((bad * e)[:e + 1], dtype=I32, device="cuda")
            for activation in ("none", "gelu"):
                y, dx, dw, db = Guarded(rows, n), Guarded(rows, k), Guarded(e, n, k), Guarded(e, n, dtype=F32)
                own = api._operators()
                scratch = torch.full((1 << 22,), 0xA5, dtype=torch.uint8, device="cuda")
                needs = []
                real = own.scratch

                def tight(need, given, device):                              # as much as is asked for, and no more
                    needs.append(need)
                    return scratch, scratch.data_ptr() + 4096, need

                own.scratch = tight
                try:
                    api.experts_forward(x, w, offsets, activation=activation, out=y.t)
                    api.experts_backward(dy, x, w, offsets, pre, activation, dx=dx.t, dw=dw.t, dbias=db.t)
                finally:
                    own.scratch = real
                torch.cuda.synchronize()
                assert all(t.intact() for t in (y, dx, dw, db))
                assert 4096 + max(needs) <= scratch.numel() and bool((scratch[:4096] == 0xA5).all()) and bool((scratch[4096 + max(needs):] == 0xA5).all())
