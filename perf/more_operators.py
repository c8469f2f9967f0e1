"""Workloads of a block of experts in a training or serving step, and of gradient clipping: the router
(choice, weights, order of the rows, gradient), moving rows to their experts and back, the products
grouped by expert (forward and backward), and the global gradient norm with clipping.

``own`` chooses what ``run`` computes: the plain form in elementary torch operations, in 32 bits and
rounded once at the end, or the library's operators (``paper_2112_01075_b200.api``).
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTIVATIONS = ("none", "relu", "gelu", "silu")
EPS = 1e-6

# the largest of each kind; drawn cases stay at or below these amounts of work
MOST_ROUTE = 16384 * 128
MOST_MOVE = 16384 * 3 * 4096
MOST_EXPERTS = 32768 * 4096 * 4096
MOST_EXPERTS_GRAD = 8192 * 4096 * 4096
MOST_WEIGHTS = 64 * 2048 * 2048
MOST_CLIP = 1 << 29


def listed():
    return [
        # the router of one decoding step: sixteen streams, one token each; latency
        dict(name="route served tokens", kind="route", type="f32", tokens=16, experts=64, k=4, normalize=True, masked=0.0, grad=False),
        # the router of a training step over [8, 2048] tokens, a few of them padding, and its gradient
        dict(name="route training step", kind="route", type="bf16", tokens=16384, experts=128, k=8, normalize=True, masked=0.03, grad=True),
        # one token of each of sixteen streams to its experts and back: latency
        dict(name="rows served tokens", kind="move", type="bf16", tokens=16, k=4, cols=4096, masked=0.0, residual=True, grad=False),
        # the [8, 2048, 4096] activations to two experts each and back, forward and backward
        dict(name="rows training step", kind="move", type="bf16", tokens=16384, k=2, cols=4096, masked=0.0, residual=True, grad=True),
        # one token at its two experts: bound by reading the two weights
        dict(name="experts one token", kind="experts", type="bf16", rows=2, experts=8, inner=4096, outer=4096,
             activation="silu", bias=False, pre=False, used=1.0, skew=0.0),
        # sixty-four streams at four of many small experts each: a few rows for every expert
        dict(name="experts served batch", kind="experts", type="bf16", rows=256, experts=64, inner=2048, outer=1024,
             activation="gelu", bias=True, pre=False, used=1.0, skew=0.5),
        # the [8, 2048, 4096] activations at two experts each, uneven shares: the largest call
        dict(name="experts activations", kind="experts", type="bf16", rows=32768, experts=8, inner=4096, outer=4096,
             activation="gelu", bias=True, pre=False, used=1.0, skew=0.5),
        # odd sizes, none of whose rows starts on a 16-byte boundary, with room behind the last expert's rows; keeps the pre-activation
        dict(name="experts odd", kind="experts", type="f16", rows=1500, experts=5, inner=1021, outer=771,
             activation="silu", bias=True, pre=True, used=0.9, skew=1.0),
        # the backward pass for one virtual device's share of the activations
        dict(name="experts gradient", kind="experts_grad", type="bf16", rows=8192, experts=8, inner=4096, outer=4096,
             activation="gelu", used=1.0, skew=0.5),
        # the backward pass at odd sizes, with rows that belong to no expert
        dict(name="experts gradient odd", kind="experts_grad", type="f16", rows=777, experts=7, inner=770, outer=1001,
             activation="silu", used=0.9, skew=1.0),
        # the gradients of the residual blocks that the training example runs (d 256, f 1024, four blocks), below the bound
        dict(name="clip blocks", kind="clip", type="mixed", tensors=24, most=262144, clip=False),
        # a layer stack's gradients: large matrices and small vectors, above the bound
        dict(name="clip large", kind="clip", type="bf16", tensors=48, most=1 << 26, clip=True),
    ]


def _size(rng, lo, hi):
    """A size whose logarithm is spread evenly; a third are multiples of 64, a third of 8, the rest any."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    grain = rng.choice((64, 8, 1))
    return max(lo, min(hi, (n + grain - 1) // grain * grain)) if n >= grain else n


def draw(rng):
    kind = rng.choice(("route", "move", "experts", "experts", "experts_grad", "clip"))
    if kind == "route":
        while True:
            t, e = _size(rng, 1, 65536), _size(rng, 2, 512)
            if t * e <= MOST_ROUTE:
                return dict(kind=kind, type=rng.choice(("bf16", "f16", "f32")), tokens=t, experts=e, k=min(e, rng.choice((1, 2, 3, 4, 6, 8))),
                            normalize=rng.random() < 0.6, masked=rng.choice((0.0, 0.1)), grad=rng.random() < 0.5)
    if kind == "move":
        while True:
            t, c, k = _size(rng, 1, 65536), _size(rng, 64, 8192), rng.choice((1, 2, 3, 4, 6, 8))
            if t * (k + 1) * c <= MOST_MOVE:
                return dict(kind=kind, type=rng.choice(("bf16", "bf16", "f16", "f32")), tokens=t, k=k, cols=c,
                            masked=rng.choice((0.0, 0.1)), residual=rng.random() < 0.5, grad=rng.random() < 0.5)
    if kind == "clip":
        return dict(kind=kind, type=rng.choice(("bf16", "f16", "f32", "mixed")), tensors=_size(rng, 1, 600), most=_size(rng, 64, 1 << 22),
                    clip=rng.random() < 0.7)
    grad = kind == "experts_grad"
    while True:
        r, e, k, n = _size(rng, 1, 32768), _size(rng, 1, 128), _size(rng, 64, 8192), _size(rng, 64, 8192)
        if r * k * n <= (MOST_EXPERTS_GRAD if grad else MOST_EXPERTS) and e * n * k <= MOST_WEIGHTS:
            break
    case = dict(kind=kind, type=rng.choice(("bf16", "f16")), rows=r, experts=e, inner=k, outer=n, activation=rng.choice(ACTIVATIONS),
                used=rng.choice((1.0, 1.0, 0.8)), skew=rng.choice((0.0, 0.5, 1.5)))
    if not grad:
        case.update(bias=rng.random() < 0.6, pre=rng.random() < 0.3)
    return case


def _counts(case, seed):
    """How many rows each expert gets: draws from uneven shares."""
    g = torch.Generator()
    g.manual_seed(int(seed) + 77)
    e, used = case["experts"], max(1, int(case["rows"] * case["used"]))
    if used <= e and case["skew"] == 0:                      # one token: different experts
        share = torch.randperm(e, generator=g)[:used]
    else:
        share = torch.multinomial(torch.softmax(torch.randn(e, generator=g) * case["skew"], 0), used, replacement=True, generator=g)
    return torch.bincount(share, minlength=e).tolist()


def _lengths(case):
    """Sizes of the gradients: a quarter of them matrices of the largest size, then smaller ones and vectors."""
    most, out = case["most"], []
    for i in range(case["tensors"]):
        out.append(max(1, (most, most // 4, max(1, most // 1024), 1 + (most // 64) * (i % 7) // 7)[i % 4]))
    while sum(out) > MOST_CLIP:
        out.pop()
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, scale=1.0, type=torch.float32):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(type)

    t, kind = TYPES.get(case["type"]), case["kind"]
    s = dict(case)
    if kind == "route":
        n, e = case["tokens"], case["experts"]
        s["logits"] = (normal(n, e) + normal(e, scale=0.5)).to(t)                # some experts are liked better than others
        s["logits"][torch.rand(n, generator=g, device="cuda") < case["masked"]] = -math.inf      # padding goes nowhere
        s["dw"] = normal(n, case["k"])
    elif kind == "move":
        n, k, c = case["tokens"], case["k"], case["cols"]
        place = torch.randperm(n * k, generator=g, device="cuda").view(n, k)
        # in the order of the experts, a token's first choices lie in token order over a few long runs
        place = place.sort(0).values.to(torch.int32)
        place[torch.rand(n, generator=g, device="cuda") < case["masked"]] = -1
        s["position"] = place
        s["weights"] = torch.softmax(normal(n, k), 1)
        s["x"] = normal(n, c, type=t)
        s["r"] = normal(n, c, type=t) if case["residual"] else None
        s["rows"] = normal(n * k, c, type=t)                                     # what the experts answered
        s["sent"] = torch.zeros((n * k, c), dtype=t, device="cuda")
        if case["grad"]:
            s["dy"] = normal(n, c, scale=n ** -0.5, type=t)
            s["back"] = torch.zeros((n * k, c), dtype=t, device="cuda")
    elif kind in ("experts", "experts_grad"):
        m, e, k, n = case["rows"], case["experts"], case["inner"], case["outer"]
        s["counts"] = _counts(case, seed)
        s["offsets"] = torch.tensor([0] + s["counts"]).cumsum(0).to(torch.int32).cuda()
        s["x"] = normal(m, k, type=t)
        s["w"] = torch.empty((e, n, k), dtype=t, device="cuda")
        for i in range(e):
            s["w"][i] = normal(n, k, scale=k ** -0.5, type=t)
        if kind == "experts":
            s["b"] = normal(e, n, scale=0.1, type=t) if case["bias"] else None
            s["y"] = torch.zeros((m, n), dtype=t, device="cuda")                 # rows of no expert are left as they are
            s["z"] = torch.zeros((m, n), dtype=t, device="cuda") if case["pre"] else None
        else:
            s["z"] = normal(m, n, type=t)
            s["dy"] = normal(m, n, scale=m ** -0.5, type=t)
            s["dx"] = torch.zeros((m, k), dtype=t, device="cuda")
    else:
        kinds = ("bf16", "f32", "f16") if t is None else (case["type"],)
        s["grads"] = [normal(n, scale=1e-3, type=TYPES[kinds[i % len(kinds)]]) for i, n in enumerate(_lengths(case))]
        total = math.sqrt(sum(_lengths(case))) * 1e-3                            # about what the norm will be
        s["bound"] = total * (0.25 if case["clip"] else 4.0)
        s["out"] = [torch.zeros_like(v) for v in s["grads"]] if case["clip"] else None
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


def _plain_route(s):
    t, l, k = s["logits"].dtype, s["logits"].float(), s["k"]
    n, e = l.shape
    left, chosen, values = l.clone(), [], []
    for _ in range(k):
        best = left.argmax(1, keepdim=True)
        value = left.gather(1, best)
        left.scatter_(1, best, -math.inf)
        chosen.append(torch.where(value > -math.inf, best, -1))
        values.append(value)
    experts, value = torch.cat(chosen, 1), torch.cat(values, 1)
    some = experts >= 0
    top = value[:, :1]
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    part = torch.exp(value - top)
    every = torch.exp(l - top)
    total = (part if s["normalize"] else every).sum(1, keepdim=True)
    weights = torch.where(some, part / torch.where(total > 0, total, torch.ones_like(total)), torch.zeros_like(part))
    flat = torch.where(some, experts, e).reshape(-1)
    order = torch.argsort(flat, stable=True)
    position = torch.empty_like(order)
    position[order] = torch.arange(n * k, device=l.device)
    position = torch.where(some, position.view(n, k), -1)
    count = (flat[:, None] == torch.arange(e, device=l.device)).sum(0)
    offsets = torch.cat([torch.zeros(1, dtype=count.dtype, device=l.device), count.cumsum(0)])
    out = {"weights": weights, "experts": experts.int(), "position": position.int(), "offsets": offsets.int()}
    if s["grad"]:
        dw = torch.where(some, s["dw"], torch.zeros_like(weights))
        mean = (weights * dw).sum(1, keepdim=True)
        at = experts.clamp(min=0)
        if s["normalize"]:
            dl = torch.zeros_like(l).scatter_add(1, at, weights * (dw - mean))
        else:
            p = every / torch.where(total > 0, total, torch.ones_like(total))
            dl = torch.zeros_like(l).scatter_add(1, at, weights * dw) - p * mean
        out["dlogits"] = dl.to(t)
    return out


def _plain_move(s):
    t, position = s["x"].dtype, s["position"].long()
    some, at = (position >= 0), position.clamp(min=0)
    sent = torch.zeros_like(s["rows"])
    sent[position[some]] = s["x"][:, None, :].expand(-1, s["k"], -1)[some]
    y = torch.zeros(s["x"].shape, device="cuda") if s["r"] is None else s["r"].float()
    weights = torch.where(some, s["weights"], torch.zeros_like(s["weights"]))
    for j in range(s["k"]):
        y = y + weights[:, j:j + 1] * s["rows"][at[:, j]].float()
    out = {"sent": sent, "y": y.to(t)}
    if s["grad"]:
        dy = s["dy"].float()
        back, dw, dx = torch.zeros_like(s["rows"]), [], torch.zeros_like(dy)
        for j in range(s["k"]):
            here = some[:, j]
            back[position[here, j]] = (weights[:, j:j + 1] * dy)[here].to(t)
            dw.append((dy * s["rows"][at[:, j]].float()).sum(1) * here)
        for j in range(s["k"]):
            dx = dx + back[at[:, j]].float() * some[:, j:j + 1]
        out.update(back=back, dw=torch.stack(dw, 1), dx=dx.to(t))
    return out


def _plain_experts(s):
    t = s["x"].dtype
    if s["kind"] == "experts":
        y = torch.zeros(s["y"].shape, device="cuda")
        z = torch.zeros(s["y"].shape, device="cuda") if s["pre"] else None
        at = 0
        for i, c in enumerate(s["counts"]):
            part = s["x"][at:at + c].float() @ s["w"][i].float().mT
            if s["b"] is not None:
                part = part + s["b"][i].float()
            if s["pre"]:
                z[at:at + c] = part
            y[at:at + c] = _activate(part, s["activation"])
            at += c
        return {"y": y.to(t), "z": z.to(t)} if s["pre"] else {"y": y.to(t)}
    dz = s["dy"].float()
    if s["activation"] != "none":
        dz = dz * _slope(s["z"].float(), s["activation"])
    dx = torch.zeros(s["x"].shape, device="cuda")
    dw, db = torch.empty(s["w"].shape, dtype=t, device="cuda"), torch.empty(s["w"].shape[:2], device="cuda")
    at = 0
    for i, c in enumerate(s["counts"]):
        part = dz[at:at + c]
        dx[at:at + c] = part @ s["w"][i].float()
        dw[i] = (part.mT @ s["x"][at:at + c].float()).to(t)
        db[i] = part.sum(0)
        at += c
    return {"dx": dx.to(t), "dw": dw, "db": db}


def _plain_clip(s):
    total = torch.zeros((), device="cuda", dtype=torch.float64)
    for v in s["grads"]:
        total = total + (v.float() * v.float()).sum()
    norm = total.sqrt().float()
    factor = torch.clamp(s["bound"] / (norm + EPS), max=1.0)
    return {"norm": norm, "grads": [(v.float() * factor).to(v.dtype) for v in s["grads"]]}


def _plain(s):
    return {"route": _plain_route, "move": _plain_move, "experts": _plain_experts, "experts_grad": _plain_experts, "clip": _plain_clip}[s["kind"]](s)


def _own(s):
    from paper_2112_01075_b200 import api
    kind = s["kind"]
    if kind == "route":
        weights, experts, position, offsets = api.route_forward(s["logits"], s["k"], normalize=s["normalize"])
        out = {"weights": weights, "experts": experts, "position": position, "offsets": offsets}
        if s["grad"]:
            out["dlogits"] = api.route_backward(s["dw"], s["logits"], weights, experts, normalize=s["normalize"])
        return out
    if kind == "move":
        sent = api.dispatch_forward(s["x"], s["position"], out=s["sent"])
        y = api.combine_forward(s["rows"], s["position"], s["weights"], residual=s["r"])
        out = {"sent": sent, "y": y}
        if s["grad"]:
            back, dw = api.combine_backward(s["dy"], s["rows"], s["position"], s["weights"], drows=s["back"])
            out.update(back=back, dw=dw, dx=api.dispatch_backward(back, s["position"]))
        return out
    if kind == "experts":
        y = api.experts_forward(s["x"], s["w"], s["offsets"], bias=s["b"], activation=s["activation"], out=s["y"], pre=s["z"])
        return {"y": y, "z": s["z"]} if s["pre"] else {"y": y}
    if kind == "experts_grad":
        dx, dw, db = api.experts_backward(s["dy"], s["x"], s["w"], s["offsets"], pre=s["z"], activation=s["activation"], dx=s["dx"])
        return {"dx": dx, "dw": dw, "db": db}
    norm = api.clip_gradients(s["grads"], s["bound"], eps=EPS, out=s["out"])
    return {"norm": norm, "grads": s["out"] if s["clip"] else s["grads"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    kind, e = case["kind"], 4 if case["type"] == "f32" else 2
    if kind == "route":
        n, m, k = case["tokens"], case["experts"], case["k"]
        b = n * m * e + 12 * n * k + 4 * (m + 1) + (n * m * e + 4 * n * k if case["grad"] else 0)
        return {"bytes": b, "flops": n * m * (4 + k) * (2 if case["grad"] else 1)}
    if kind == "move":
        n, k, c = case["tokens"], case["k"], case["cols"]
        rows = 1 + k + k + 1 + case["residual"]                  # x in, rows out; rows in, y out
        if case["grad"]:
            rows += 1 + k + k + k + 1                            # dy and rows in, their gradient out; that in, dx out
        return {"bytes": rows * n * c * e + 8 * n * k, "flops": 2 * n * k * c * (4 if case["grad"] else 1)}
    if kind in ("experts", "experts_grad"):
        m, k, n = case["rows"], case["inner"], case["outer"]
        used = max(1, int(m * case["used"]))
        busy = min(case["experts"], used) * n * k                # weights of experts that have rows
        if kind == "experts":
            return {"bytes": (busy + used * (k + n * (1 + case["pre"]))) * e, "flops": 2 * used * n * k}
        b = busy + case["experts"] * n * k + used * (n * (1 if case["activation"] == "none" else 2) + 2 * k)
        return {"bytes": b * e + 4 * case["experts"] * n, "flops": 4 * used * n * k}
    sizes = _lengths(case)
    kinds = (2, 4, 2) if case["type"] == "mixed" else (e,)
    b = sum(n * kinds[i % len(kinds)] for i, n in enumerate(sizes))
    return {"bytes": b * (2 if case["clip"] else 1), "flops": sum(sizes) * (3 if case["clip"] else 2)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "route":
        l, k = s["logits"].double(), case["k"]
        n, e = l.shape
        ranked = torch.sort(l, dim=1, descending=True, stable=True)
        value, experts = ranked.values[:, :k], ranked.indices[:, :k]
        some = value != -math.inf
        base = torch.logsumexp(value if case["normalize"] else l, dim=1, keepdim=True)
        weights = torch.exp(value - base).masked_fill(~some, 0.0)
        experts = experts.masked_fill(~some, -1)
        # a row's place: the rows of lower experts, and those of the same expert before it
        hit = torch.zeros((n, e), dtype=torch.int64, device="cuda")
        token = torch.arange(n, device="cuda")[:, None].expand(n, k)
        hit[token[some], experts[some]] = 1
        total = hit.sum(0)
        offsets = torch.nn.functional.pad(total.cumsum(0), (1, 0))
        before = hit.cumsum(0) - hit
        position = torch.full((n, k), -1, dtype=torch.int64, device="cuda")
        position[some] = (before + offsets[:-1])[token[some], experts[some]]
        out = {"weights": weights, "experts": experts.int(), "position": position.int(), "offsets": offsets.int()}
        if case["grad"]:
            dw = s["dw"].double().masked_fill(~some, 0.0)
            dp = torch.zeros((n, e), dtype=torch.float64, device="cuda")
            dp[token[some], experts[some]] = dw[some]
            p = torch.exp(l - base).masked_fill(~some.any(1, keepdim=True), 0.0)
            if case["normalize"]:
                p = p * hit
            out["dlogits"] = p * (dp - (p * dp).sum(1, keepdim=True))
        return out
    if kind == "move":
        # the moves as one sparse matrix [tokens, rows] of ones or weights
        n, k, c = case["tokens"], case["k"], case["cols"]
        some = s["position"] >= 0
        token = torch.arange(n, device="cuda")[:, None].expand(n, k)[some]
        row, w = s["position"][some].long(), s["weights"].double()[some]
        sent = torch.zeros((n * k, c), dtype=torch.float64, device="cuda")
        sent.index_copy_(0, row, s["x"].double().index_select(0, token))
        y = torch.zeros((n, c), dtype=torch.float64, device="cuda") if s["r"] is None else s["r"].double()
        y = y.index_add(0, token, s["rows"].double().index_select(0, row) * w[:, None])
        out = {"sent": sent, "y": y}
        if case["grad"]:
            del sent, y
            dy = s["dy"].double().index_select(0, token)
            out["back"] = torch.zeros((n * k, c), dtype=torch.float64, device="cuda").index_copy_(0, row, dy * w[:, None])
            dw = torch.zeros((n, k), dtype=torch.float64, device="cuda")
            dw[some] = torch.linalg.vecdot(dy, s["rows"].double().index_select(0, row))
            out["dw"] = dw
            out["dx"] = s["dy"].double() * torch.where(some, s["weights"].double(), 0.0).sum(1, keepdim=True)
        return out
    if kind in ("experts", "experts_grad"):
        m, e = case["rows"], case["experts"]
        ends = s["offsets"].tolist()
        act = case["activation"]
        if kind == "experts":
            y = torch.zeros((m, case["outer"]), dtype=torch.float64, device="cuda")
            z = torch.zeros_like(y)
            for i in range(e):
                here = slice(ends[i], ends[i + 1])
                v = torch.nn.functional.linear(s["x"][here].double(), s["w"][i].double(), None if s["b"] is None else s["b"][i].double())
                z[here] = v
                if act == "relu":
                    v = torch.where(v > 0, v, 0.0)
                elif act == "gelu":
                    v = v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
                elif act == "silu":
                    v = v / (1 + torch.exp(-v))
                y[here] = v
            return {"y": y, "z": z} if case["pre"] else {"y": y}
        dz, z = s["dy"].double(), s["z"].double()
        if act == "relu":
            dz = torch.where(z > 0, dz, 0.0)
        elif act == "gelu":
            dz = dz * (0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        elif act == "silu":
            q = 1 / (1 + torch.exp(-z))
            dz = dz * (q + z * q * (1 - q))
        dx = torch.zeros((m, case["inner"]), dtype=torch.float64, device="cuda")
        dw, db = torch.zeros(s["w"].shape, dtype=torch.float64, device="cuda"), torch.zeros((e, case["outer"]), dtype=torch.float64, device="cuda")
        for i in range(e):
            here = slice(ends[i], ends[i + 1])
            dx[here] = torch.mm(dz[here], s["w"][i].double())
            dw[i] = torch.einsum("tn,tk->nk", dz[here], s["x"][here].double())
            db[i] = torch.einsum("tn->n", dz[here])
        return {"dx": dx, "dw": dw, "db": db}
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(v.double()) for v in s["grads"]]))
    factor = min(1.0, s["bound"] / (float(norm) + EPS))
    return {"norm": norm, "grads": [v.double() * factor for v in s["grads"]]}
