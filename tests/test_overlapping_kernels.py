"""Kernels that are started while the one before them in the stream still runs read what that one writes.

A load from the read-only path (``__ldg``, ``ld.global.nc``) takes for granted that nobody writes there during the lifetime of
the kernel, the time included in which it waits; a plain load does not.  A run of calls cannot show that no such load comes
too early, so the sources are looked through; the runs that follow chain calls over buffers that are used again and again,
and compare every result, bit by bit, with that of the same calls with a pause between them.
"""
import glob
import os
import re

import numpy as np
import pytest

import oracle
from paper_2112_01075_b200 import api

torch = pytest.importorskip("torch")

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
CSRC = os.path.join(os.path.dirname(api.__file__), "csrc")
WAITS = re.compile(r"\bwait_for_previous(_kernel)?\(\)")


def code_of(path):
    text = open(path).read()
    return re.sub(r"/\*.*?\*/", "", re.sub(r"//[^\n]*", "", text), flags=re.S)


def sources_that_wait():
    kernels = [p for p in sorted(glob.glob(os.path.join(CSRC, "*.cu"))) if WAITS.search(code_of(p))]
    return kernels + sorted(glob.glob(os.path.join(CSRC, "*.cuh")))


@pytest.mark.parametrize("path", sources_that_wait(), ids=os.path.basename)
def test_no_load_takes_the_read_only_path(path):
    found = [line for line in code_of(path).splitlines() if re.search(r"__ldg\b|\.nc\b|__ldlu\b|__restrict__", line)]
    assert not found, found


def test_the_sources_of_all_kernels_are_looked_through():
    names = {os.path.basename(p) for p in sources_that_wait()}
    assert {"kernels.cu", "few.cu", "rows.cu", "product.cu", "experts.cu", "routing.cu", "clip.cu", "elements.cuh", "activation.cuh"} <= names


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rand(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def back_to_back(calls, results, turns):
    """Runs ``calls(i, pause)`` for every turn, first with a pause after each call, then without; the results have to agree."""
    def pause():
        torch.cuda.synchronize()
    want = []
    for i in range(turns):
        calls(i, pause)
        torch.cuda.synchronize()
        want.append([t.clone() for t in results])
    got = []
    for i in range(turns):
        calls(i, lambda: None)
        got.append([t.clone() for t in results])
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(want, got)):
        assert all(torch.equal(u, v) for u, v in zip(a, b)), i
    return want


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,d,f", [(1, 1024, 4096), (8, 512, 520), (9, 4096, 256), (16, 1000, 333), (32, 256, 1024), (31, 129, 70)])
def test_layer_norm_and_linear_layers_of_a_few_rows(rows, d, f, dtype):
    """norm, first layer, second layer, all into the same buffers every time; the weight is one of the buffers too."""
    g = gen(rows + d)
    inputs = [rand(g, rows, d, dtype=dtype) for _ in range(6)]
    gamma, beta = rand(g, d), rand(g, d)
    stored = [rand(g, f, d, dtype=dtype, scale=d ** -0.5) for _ in range(2)]
    w1, w2 = torch.empty_like(stored[0]), rand(g, d, f, dtype=dtype, scale=f ** -0.5)
    n, u, y = torch.empty_like(inputs[0]), torch.empty((rows, f), dtype=dtype, device="cuda"), torch.empty_like(inputs[0])
    places = torch.arange(f, device="cuda", dtype=torch.int32).view(f, 1)

    def calls(i, pause):
        api.dispatch_forward(stored[i % 2], places, out=w1)                 # a weight that a kernel has just written
        pause()
        api.layer_norm_forward(inputs[i % 6], gamma, beta, out=n)
        pause()
        api.linear_forward(n, w1, activation="gelu", out=u)
        pause()
        api.linear_forward(u, w2, residual=n, out=y)
    want = back_to_back(calls, [n, u, y], 24)
    assert not torch.equal(want[0][2], want[1][2])


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cols", [(4096, 96), (3000, 1024), (700, 2047)])
def test_sums_over_rows_behind_what_they_add(rows, cols):
    """Gradients whose sums are added by a kernel of their own from parts in a scratch that is used again."""
    g = gen(rows)
    inputs = [rand(g, rows, cols, dtype=BF16) for _ in range(4)]
    dy, gamma, beta = rand(g, rows, cols, dtype=BF16), rand(g, cols), rand(g, cols)
    w = rand(g, 64, cols, dtype=BF16)
    dz = [rand(g, rows, 64, dtype=BF16) for _ in range(4)]
    scratch = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    kept = [api.layer_norm_forward(x, gamma, beta) for x in inputs]
    dgamma, dbeta, db = torch.empty_like(gamma), torch.empty_like(beta), torch.empty(64, device="cuda")
    dx = torch.empty_like(dy)

    def calls(i, pause):
        _, mean, scale = kept[i % 4]
        got = api.layer_norm_backward(dy, inputs[i % 4], gamma, mean, scale, scratch=scratch)
        pause()
        dx.copy_(got[0])
        dgamma.copy_(got[1])
        dbeta.copy_(got[2])
        pause()
        db.copy_(api.linear_backward(dz[i % 4], inputs[i % 4], w, scratch=scratch)[2])
    back_to_back(calls, [dx, dgamma, dbeta, db], 12)


@pytest.mark.gpu
@pytest.mark.parametrize("n,m", [(256, 256), (512, 2048), (200, 328)])
def test_orthogonalisation_of_what_a_product_has_written(n, m):
    g = gen(n + m)
    a, b = [rand(g, n, 512, dtype=BF16) for _ in range(3)], rand(g, m, 512, dtype=BF16, scale=512 ** -0.5)
    x, out = torch.empty((n, m), dtype=BF16, device="cuda"), torch.empty((n, m), dtype=BF16, device="cuda")

    def calls(i, pause):
        api.linear_forward(a[i % 3], b, out=x)
        pause()
        api.orthogonalize(x, out=out)
    back_to_back(calls, [x, out], 9)


MOVES = [  # mesh, source, target, bytes of an element, mode: several launches, and runs of few bytes, ragged or interleaved
    ((2, 3, 2), ((12, 12, 8), ((0,), (1,), ())), ((12, 12, 8), ((1,), (), (0,))), 4, api.FUSE_NONE),
    ((4, 2), ((8 * 37, 8 * 101), ((0,), (1,))), ((8 * 37, 8 * 101), ((1,), (0,))), 2, api.NAIVE),
    ((4,), ((36, 44, 28), ((0,), (), ())), ((36, 44, 28), ((), (), (0,))), 2, api.FUSE_ADJACENT),
    ((4, 4, 4), ((8, 12, 4, 28, 20, 12), ((), (1,), (), (2,), (), ())), ((8, 12, 4, 28, 20, 12), ((2,), (), (), (), (0,), (1,))), 4, api.FUSE_NONE),
    ((2, 3), ((30, 66), ((0,), (1,))), ((30, 66), ((1,), (0,))), 1, api.FUSE_NONE),
]


@pytest.mark.gpu
@pytest.mark.parametrize("mesh,src,dst,e,mode", MOVES)
def test_redistributions_one_after_the_other(mesh, src, dst, e, mode):
    """There and back again over the same tiles, with other data every time that a kernel has written just before."""
    there, back = api.Plan(mesh, src, dst, e, mode), api.Plan(mesh, dst, src, e, mode)
    n = there.n_devices
    rng = np.random.default_rng(n + e)
    arrays = [rng.integers(0, 256, size=src[0] + (e,), dtype=np.uint8) for _ in range(3)]
    stored = [[torch.from_numpy(np.ascontiguousarray(t).reshape(-1)).cuda() for t in oracle.reslice(mesh, src, a)] for a in arrays]
    wanted = [[torch.from_numpy(np.ascontiguousarray(t).reshape(-1)).cuda() for t in oracle.reslice(mesh, dst, a)] for a in arrays]
    a, b, c = ([torch.zeros(p.local_elems(i) * e, dtype=torch.uint8, device="cuda") for _ in range(n)] for p, i in ((there, 0), (there, 1), (back, 1)))
    spaces = there.alloc_scratch(), back.alloc_scratch()
    for i in range(30):
        for t, s in zip(a, stored[i % 3]):
            t.copy_(s)
        there.execute(a, b, spaces[0])
        back.execute(b, c, spaces[1])
        there.execute(c, b, spaces[0])
        back.execute(b, a, spaces[1])
        there.execute(a, b, spaces[0])
        got = [t.clone() for t in a], [t.clone() for t in b], [t.clone() for t in c]
        assert all(torch.equal(x, y) for x, y in zip(got[0], stored[i % 3])) and all(torch.equal(x, y) for x, y in zip(got[2], stored[i % 3]))
        assert all(torch.equal(x, y) for x, y in zip(got[1], wanted[i % 3])), i
