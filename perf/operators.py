"""Workloads of the operators that run on a device's tiles between two redistributions: the linear
layer with its epilogue (forward and backward), layer norm (forward and backward) and the
orthogonalisation of a weight update by Newton-Schulz products.

``own`` chooses what ``run`` computes: the plain form in elementary torch operations, in 32 bits and
rounded once at the end, or the library's operators (``paper_2112_01075_b200.api``).
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTIVATIONS = ("none", "relu", "gelu", "silu")
STEPS, COEFFICIENTS, NORM_EPS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7, 1e-5

# the largest of each kind; drawn cases stay at or below these amounts of work
MOST_LINEAR = 16384 * 4096 * 16384
MOST_LINEAR_GRAD = 4096 * 4096 * 16384
MOST_NORM = 16384 * 4096
MOST_ORTHOGONALIZE = 8 * 2048 ** 3


def listed():
    return [
        # one token of a served stream through a square projection: the smallest call, bound by reading the weight
        dict(name="linear one row", kind="linear", type="bf16", rows=1, inner=4096, outer=4096,
             activation="none", bias=True, residual=True, pre=False),
        # a small batch of tokens through the wide projection of a feed-forward block
        dict(name="linear few rows", kind="linear", type="bf16", rows=24, inner=4096, outer=16384,
             activation="gelu", bias=True, residual=False, pre=False),
        # the [8, 2048, 4096] activations of the reshard benchmark through the wide projection: the largest call
        dict(name="linear activations", kind="linear", type="bf16", rows=16384, inner=4096, outer=16384,
             activation="gelu", bias=True, residual=False, pre=False),
        # odd sizes, none of whose rows starts on a 16-byte boundary; a training forward that keeps the pre-activation
        dict(name="linear odd", kind="linear", type="f16", rows=1000, inner=1021, outer=2047,
             activation="silu", bias=True, residual=True, pre=True),
        # the backward pass of the wide projection for one virtual device's share of the activations
        dict(name="linear gradient", kind="linear_grad", type="bf16", rows=4096, inner=4096, outer=16384,
             activation="gelu"),
        # the backward pass at odd sizes
        dict(name="linear gradient odd", kind="linear_grad", type="f16", rows=333, inner=770, outer=1001,
             activation="silu"),
        # the [8, 2048, 4096] activations, normalised before a projection
        dict(name="norm activations", kind="norm", type="bf16", rows=16384, cols=4096),
        # three tokens of a served stream in 32 bits: latency
        dict(name="norm three rows", kind="norm", type="f32", rows=3, cols=4096),
        # the backward pass of the same activations, with the reduction of the weight's gradient over all rows
        dict(name="norm gradient", kind="norm_grad", type="bf16", rows=16384, cols=4096),
        # an odd row length in 32 bits: rows that start on 4-byte boundaries only
        dict(name="norm gradient odd", kind="norm_grad", type="f32", rows=2047, cols=1531),
        # the share of a virtual device in a stack of square weights whose updates are orthogonalised
        dict(name="orthogonalize stack", kind="orthogonalize", type="bf16", batch=8, rows=2048, cols=2048),
        # one odd tall momentum matrix held in 32 bits
        dict(name="orthogonalize odd", kind="orthogonalize", type="f32", batch=1, rows=1111, cols=520),
    ]


def _size(rng, lo, hi):
    """A size whose logarithm is spread evenly; a third are multiples of 64, a third of 8, the rest any."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    grain = rng.choice((64, 8, 1))
    return max(lo, min(hi, (n + grain - 1) // grain * grain)) if n >= grain else n


def draw(rng):
    kind = rng.choice(("linear", "linear", "linear_grad", "norm", "norm_grad", "orthogonalize"))
    if kind in ("linear", "linear_grad"):
        grad = kind == "linear_grad"
        while True:
            m, k, n = _size(rng, 16 if grad else 1, 16384), _size(rng, 64, 16384), _size(rng, 64, 16384)
            if m * k * n <= (MOST_LINEAR_GRAD if grad else MOST_LINEAR):
                break
        case = dict(kind=kind, type=rng.choice(("bf16", "f16")), rows=m, inner=k, outer=n,
                    activation=rng.choice(ACTIVATIONS))
        if not grad:
            case.update(bias=rng.random() < 0.7, residual=rng.random() < 0.4, pre=rng.random() < 0.3)
        return case
    if kind in ("norm", "norm_grad"):
        while True:
            m, c = _size(rng, 1, 65536), _size(rng, 64, 16384)
            if m * c <= MOST_NORM:
                return dict(kind=kind, type=rng.choice(("bf16", "f16", "f32")), rows=m, cols=c)
    while True:
        batch, m, n = _size(rng, 1, 32), _size(rng, 32, 4096), _size(rng, 32, 8192)
        if batch * min(m, n) ** 2 * max(m, n) <= MOST_ORTHOGONALIZE:
            return dict(kind=kind, type=rng.choice(("bf16", "f16", "f32")), batch=batch, rows=m, cols=n)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, scale=1.0, type=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(type)

    t, kind = TYPES[case["type"]], case["kind"]
    s = dict(case)
    if kind in ("linear", "linear_grad"):
        m, k, n = case["rows"], case["inner"], case["outer"]
        s["x"] = normal(m, k, type=t)
        s["w"] = normal(n, k, scale=k ** -0.5, type=t)
        if kind == "linear":
            s["b"] = normal(n, scale=0.1, type=t) if case["bias"] else None
            s["r"] = normal(m, n, type=t) if case["residual"] else None
        else:
            s["z"] = normal(m, n, type=t)                       # the pre-activation that the forward pass kept
            s["dy"] = normal(m, n, scale=m ** -0.5, type=t)
    elif kind in ("norm", "norm_grad"):
        r, c = case["rows"], case["cols"]
        columns = torch.exp(normal(c, scale=0.5))               # some channels are larger than others ...
        rows = normal(r, 1, scale=0.5)                          # ... and a row's mean is not zero
        s["x"] = (normal(r, c) * columns + rows).to(t)
        s["g"] = 1 + normal(c, scale=0.1)
        s["b"] = normal(c, scale=0.1)
        if kind == "norm_grad":
            s["dy"] = normal(r, c, scale=r ** -0.5, type=t)
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + EPS)
    else:
        b, m, n = case["batch"], case["rows"], case["cols"]
        rank = max(1, min(m, n) // 16)                          # a gradient: a few strong directions over noise
        strength = torch.logspace(0, -1.5, rank, device="cuda")
        x = torch.bmm(normal(b, m, rank) * strength, normal(b, rank, n))
        s["x"] = ((x + 0.3 * normal(b, m, n)) * 1e-3).to(t)
    return s


def _activate(z, activation):
    if activation == "relu":
        return torch.clamp(z, min=0)
    if activation == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if activation == "silu":
        return z * torch.sigmoid(z)
    return z


def _slope(z, activation):
    if activation == "relu":
        return (z > 0).to(z.dtype)
    if activation == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if activation == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _plain(s):
    kind = s["kind"]
    if kind == "linear":
        t = s["x"].dtype
        z = s["x"].float() @ s["w"].float().mT
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _activate(z, s["activation"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return {"y": y.to(t), "z": z.to(t)} if s["pre"] else {"y": y.to(t)}
    if kind == "linear_grad":
        t = s["x"].dtype
        dz = s["dy"].float()
        if s["activation"] != "none":
            dz = dz * _slope(s["z"].float(), s["activation"])
        return {"dx": (dz @ s["w"].float()).to(t), "dw": (dz.mT @ s["x"].float()).to(t), "db": dz.sum(0)}
    if kind == "norm":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        d = x - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        return {"y": (d * rstd * s["g"] + s["b"]).to(s["x"].dtype), "mean": mean[:, 0], "rstd": rstd[:, 0]}
    if kind == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xh = (s["x"].float() - s["mean"][:, None]) * rstd
        c = dy * s["g"]
        dx = (c - c.mean(1, keepdim=True) - xh * (c * xh).mean(1, keepdim=True)) * rstd
        return {"dx": dx.to(s["x"].dtype), "dg": (dy * xh).sum(0), "db": dy.sum(0)}
    x = s["x"].float()
    x = x / ((x * x).sum((1, 2), keepdim=True).sqrt() + NORM_EPS)
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    a, b, c = COEFFICIENTS
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    x = x.mT if tall else x
    return {"x": x.to(torch.bfloat16).contiguous()}             # the update is bf16 whatever the input's type


def _own(s):
    from paper_2112_01075_b200 import api
    kind = s["kind"]
    if kind == "linear":
        z = torch.empty((s["rows"], s["outer"]), dtype=s["x"].dtype, device="cuda") if s["pre"] else None
        y = api.linear_forward(s["x"], s["w"], bias=s["b"], residual=s["r"], activation=s["activation"], pre=z)
        return {"y": y, "z": z} if s["pre"] else {"y": y}
    if kind == "linear_grad":
        dx, dw, db = api.linear_backward(s["dy"], s["x"], s["w"], pre=s["z"], activation=s["activation"])
        return {"dx": dx, "dw": dw, "db": db}
    if kind == "norm":
        y, mean, rstd = api.layer_norm_forward(s["x"], s["g"], s["b"], eps=EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        dx, dg, db = api.layer_norm_backward(s["dy"], s["x"], s["g"], s["mean"], s["rstd"])
        return {"dx": dx, "dg": dg, "db": db}
    return {"x": api.orthogonalize(s["x"], steps=STEPS, coefficients=COEFFICIENTS, eps=NORM_EPS)}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind, e = case["kind"], 4 if case["type"] == "f32" else 2
    if kind == "linear":
        m, k, n = case["rows"], case["inner"], case["outer"]
        b = m * k + n * k + n * case["bias"] + m * n * (1 + case["residual"] + case["pre"])
        return {"bytes": b * e, "flops": 2 * m * n * k}
    if kind == "linear_grad":
        m, k, n = case["rows"], case["inner"], case["outer"]
        b = m * n * (1 if case["activation"] == "none" else 2) + 2 * m * k + 2 * n * k
        return {"bytes": b * e + 4 * n, "flops": 4 * m * n * k}
    if kind == "norm":
        r, c = case["rows"], case["cols"]
        return {"bytes": 2 * r * c * e + 8 * c + 8 * r, "flops": 8 * r * c}
    if kind == "norm_grad":
        r, c = case["rows"], case["cols"]
        return {"bytes": 3 * r * c * e + 12 * c + 8 * r, "flops": 14 * r * c}
    b, m, n = case["batch"], *sorted((case["rows"], case["cols"]))
    # gram and its square are symmetric: half of each needs computing
    return {"bytes": b * m * n * (e + 2), "flops": STEPS * b * (m * m * n + m * m * m + 2 * m * m * n)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if kind == "linear":
        z = torch.mm(wide["x"], wide["w"].t())
        if "b" in wide:
            z += wide["b"]
        act = case["activation"]
        y = z
        if act == "relu":
            y = torch.where(z > 0, z, torch.zeros_like(z))
        elif act == "gelu":
            y = z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        elif act == "silu":
            y = z / (1 + torch.exp(-z))
        if "r" in wide:
            y = y + wide["r"]
        return {"y": y, "z": z} if case["pre"] else {"y": y}
    if kind == "linear_grad":
        z, act, dz = wide["z"], case["activation"], wide["dy"]
        if act == "relu":
            dz = torch.where(z > 0, dz, torch.zeros_like(dz))
        elif act == "gelu":
            dz = dz * (0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        elif act == "silu":
            q = 1 / (1 + torch.exp(-z))
            dz = dz * (q + z * q * (1 - q))
        return {"dx": torch.mm(dz, wide["w"]), "dw": torch.mm(dz.t(), wide["x"]), "db": dz.sum(dim=0)}
    if kind == "norm":
        var, mean = torch.var_mean(wide["x"], dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = torch.addcmul(wide["b"], (wide["x"] - mean[:, None]) * rstd[:, None], wide["g"])
        return {"y": y, "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        n = case["cols"]
        xh = (wide["x"] - wide["mean"][:, None]) * wide["rstd"][:, None]
        dxh = wide["dy"] * wide["g"]
        along = torch.einsum("rc,rc->r", dxh, xh)[:, None]
        dx = (n * dxh - dxh.sum(dim=1, keepdim=True) - xh * along) * (wide["rstd"][:, None] / n)
        return {"dx": dx, "dg": torch.einsum("rc,rc->c", wide["dy"], xh), "db": wide["dy"].sum(dim=0)}
    # the iteration as one polynomial of the Gram matrix, applied to the normalised input once
    x = wide["x"]
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + NORM_EPS)
    flip = x.shape[-2] > x.shape[-1]
    if flip:
        x = x.transpose(-1, -2)
    a, b, c = COEFFICIENTS
    one = torch.eye(x.shape[-2], dtype=torch.float64, device=x.device)
    gram, total = torch.bmm(x, x.transpose(-1, -2)), one
    for _ in range(STEPS):
        p = a * one + b * gram + c * torch.matmul(gram, gram)
        total = torch.matmul(p, total)
        gram = torch.matmul(torch.matmul(p, gram), p)
    x = torch.matmul(total, x)
    return {"x": (x.transpose(-1, -2) if flip else x).contiguous()}
