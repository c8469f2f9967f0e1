"""A training step of sharded residual blocks: the operators on the tiles, redistributions between them.

``python -m paper_2112_01075_b200.block [experts]`` trains a few blocks  y = x + gelu(norm(x) w1^T + b1) w2^T + b2  on a mesh of
four virtual devices towards random targets and prints the loss.  Nothing is summed across devices but the layer norm's
weight gradients: wherever a sum over devices would be needed, the operand is brought into the sharding in which the sum
is local.  Types (a: the mesh axis; a device's tile is what the operators see):

    activations      [rows{a}, d]   layer norm, second product with the residual, gradients of the inputs
                     [rows, f{a}]   first product: each device computes its own features
    weights          [f{a}, d], [d{a}, f]: as they are kept, and as their gradients come out
    weight updates   a stack over the blocks, [n, f{a}, d] -> [n{a}, f, d]: whole matrices, orthogonalised where they lie,
                     and back

Every redistribution is planned once and executed on lists of tiles (``api.Plan``).

:class:`ExpertBlocks` (``experts``) has a set of experts of which every token uses ``k`` in the place of the two weights.  The
``rows * k`` rows in the order of the experts are arrays of static size, so they move by the same kind of plans; only where
an expert's rows begin depends on the data, and stays on the device:

    tokens           [rows, d{a}]       dispatched and combined: each device moves its own columns
    rows by expert   [rows k, f{a}]     first product: each device computes its own features of every expert
                     [rows k{a}, d]     second product, gradients of the inputs: a device's rows are some experts' ranges
    weights          [experts, f{a}, d], [experts, d{a}, f]
    weight updates   a stack over blocks and experts
"""
from __future__ import annotations

from typing import Dict, List

from . import api


class Blocks:
    """``n`` residual blocks of width ``d`` and hidden width ``f`` over ``devices`` virtual devices, bfloat16 weights."""

    def __init__(self, n: int = 4, rows: int = 512, d: int = 256, f: int = 1024, devices: int = 4, seed: int = 0):
        torch = self._sizes(n, n, rows, d, f, devices)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        bf16 = torch.bfloat16

        def weight(out, inner):                                  # row-sharded tiles of one weight per block
            return [[(torch.randn((out // devices, inner), generator=g, device="cuda") * inner ** -0.5).to(bf16)
                     for _ in range(devices)] for _ in range(n)]

        self.w1, self.w2 = weight(f, d), weight(d, f)
        self.b1 = [[torch.zeros(f // devices, device="cuda") for _ in range(devices)] for _ in range(n)]
        self.b2 = [torch.zeros(d, device="cuda") for _ in range(n)]
        self.gamma = [torch.ones(d, device="cuda") for _ in range(n)]
        self.beta = [torch.zeros(d, device="cuda") for _ in range(n)]
        self.momentum = {"w1": [[torch.zeros_like(t, dtype=torch.float32) for t in w] for w in self.w1],
                         "w2": [[torch.zeros_like(t, dtype=torch.float32) for t in w] for w in self.w2]}

    def _sizes(self, n: int, matrices: int, rows: int, d: int, f: int, devices: int):
        """Keeps the sizes; ``matrices``: of one name in all blocks.  Returns torch."""
        import torch

        if matrices % devices or rows % devices or d % devices or f % devices:
            raise ValueError("the matrices of all blocks, rows and widths have to be divisible by the number of devices")
        self.torch, self.n, self.rows, self.d, self.f, self.devices = torch, n, rows, d, f, devices
        self.mesh = (devices,)
        self._plans: Dict = {}
        return torch

    # ---- redistributions -------------------------------------------------------------------------------

    def move(self, tiles: List, shape, src, dst) -> List:
        """``tiles`` of a global array of ``shape`` from the sharding ``src`` to ``dst``: the dimension that the mesh axis
        partitions, or None for a replicated array."""
        key = (tuple(shape), src, dst, tiles[0].element_size())
        if key not in self._plans:
            axes = lambda dim: tuple((0,) if k == dim else () for k in range(len(shape)))       # noqa: E731
            self._plans[key] = api.Plan(self.mesh, (shape, axes(src)), (shape, axes(dst)), tiles[0].element_size())
        plan = self._plans[key]
        local = [s // self.devices if k == dst else s for k, s in enumerate(shape)]
        out = [self.torch.empty(local, dtype=tiles[0].dtype, device="cuda") for _ in range(self.devices)]
        plan.execute([t.contiguous() for t in tiles], out, plan.alloc_scratch())
        return out

    # ---- one block -----------------------------------------------------------------------------------------

    def forward(self, k: int, x: List):
        """Block ``k`` on row-sharded ``x``: the row-sharded result, and what the backward pass needs."""
        R, d, f, devices = self.rows, self.d, self.f, range(self.devices)
        norms = [api.layer_norm_forward(x[i], self.gamma[k], self.beta[k]) for i in devices]
        full = self.move([y for y, _, _ in norms], (R, d), 0, None)
        z = [self.torch.empty((R, f // self.devices), dtype=x[0].dtype, device="cuda") for _ in devices]
        u = [api.linear_forward(full[j], self.w1[k][j], bias=self.b1[k][j], activation="gelu", pre=z[j]) for j in devices]
        u = self.move(u, (R, f), 1, 0)
        w2 = self.move(self.w2[k], (d, f), 0, None)
        y = [api.linear_forward(u[i], w2[i], bias=self.b2[k], residual=x[i]) for i in devices]
        return y, (x, norms, full, z, u, w2)

    def backward(self, k: int, dy: List, kept):
        """Row-sharded gradient of block ``k``'s input, and the gradients of its weights, sharded as they are."""
        x, norms, full, z, u, w2 = kept
        R, d, f, devices = self.rows, self.d, self.f, range(self.devices)
        # second product: dw2 of a device's own rows of w2 needs its columns of dy and all of u
        dy_cols, u_full = self.move(dy, (R, d), 0, 1), self.move(u, (R, f), 0, None)
        second = [api.linear_backward(dy_cols[j], u_full[j], self.w2[k][j], need=(False, True, True)) for j in devices]
        du = [api.linear_backward(dy[i], u[i], w2[i], need=(True, False, False))[0] for i in devices]
        # first product: the same, with the activation's slope
        du_cols, z_rows, w1 = self.move(du, (R, f), 0, 1), self.move(z, (R, f), 1, 0), self.move(self.w1[k], (f, d), 0, None)
        first = [api.linear_backward(du_cols[j], full[j], self.w1[k][j], z[j], "gelu", need=(False, True, True)) for j in devices]
        dn = [api.linear_backward(du[i], norms[i][0], w1[i], z_rows[i], "gelu", need=(True, False, False))[0] for i in devices]
        back = [api.layer_norm_backward(dn[i], x[i], self.gamma[k], norms[i][1], norms[i][2]) for i in devices]
        dx = [back[i][0] + dy[i] for i in devices]
        return dx, {"w1": [g[1] for g in first], "b1": [g[2] for g in first], "w2": [g[1] for g in second],
                    "b2": self.torch.cat([g[2] for g in second]), "gamma": sum(b[1] for b in back), "beta": sum(b[2] for b in back)}

    # ---- the update ------------------------------------------------------------------------------------------

    def orthogonal(self, name: str, tiles: List[List]) -> List[List]:
        """``tiles[k][j]`` (block, device), sharded on the weight's rows: the same of the orthogonalised matrices."""
        torch, (rows, cols) = self.torch, ((self.f, self.d) if name == "w1" else (self.d, self.f))
        stacks = [torch.stack([tiles[k][j] for k in range(self.n)]) for j in range(self.devices)]
        whole = self.move(stacks, (self.n, rows, cols), 1, 0)
        done = [api.orthogonalize(t, scale=max(1.0, rows / cols) ** 0.5) for t in whole]
        back = self.move(done, (self.n, rows, cols), 0, 1)
        return [[back[j][k] for j in range(self.devices)] for k in range(self.n)]

    def gradients(self, x: List, target: List):
        """Loss (mean squared error) and every block's gradients, for row-sharded input and target."""
        kept = []
        for k in range(self.n):
            x, state = self.forward(k, x)
            kept.append(state)
        error = [a.float() - b.float() for a, b in zip(x, target)]
        count = self.rows * self.d
        loss = sum((e * e).sum() for e in error) / count
        dy = [(e * (2.0 / count * self.scale)).to(x[0].dtype) for e in error]
        grads = [None] * self.n
        for k in reversed(range(self.n)):
            dy, grads[k] = self.backward(k, dy, kept[k])
        return loss, grads

    scale = 2.0 ** 12                                            # of the loss, so that bfloat16 gradients stay normal

    replicated = ("b2", "gamma", "beta")                         # parameters of which every device has the whole

    def clip(self, grads: List[Dict], bound: float):
        """Scales the gradients of all blocks, every tile of every one, down to a norm of ``bound``; returns the norm before."""
        tiles = [t for g in grads for v in g.values() for t in (v if isinstance(v, list) else [v])]
        return api.clip_gradients(tiles, bound * self.scale) / self.scale

    def step(self, x: List, target: List, rate: float = 0.02, momentum: float = 0.9, clip=None):
        """One training step, with gradients of a norm of at most ``clip`` if it is given; returns the loss before it."""
        loss, grads = self.gradients(x, target)
        if clip is not None:
            self.clip(grads, clip)
        for name, weights in (("w1", self.w1), ("w2", self.w2)):
            for k in range(self.n):
                for j in range(self.devices):
                    self.momentum[name][k][j].mul_(momentum).add_(grads[k][name][j].float())
            update = self.orthogonal(name, self.momentum[name])
            for k in range(self.n):
                for j in range(self.devices):
                    weights[k][j].sub_(update[k][j], alpha=rate)
        for k in range(self.n):
            for j in range(self.devices):
                self.b1[k][j].sub_(grads[k]["b1"][j], alpha=rate / self.scale)
            for name in self.replicated:
                getattr(self, name)[k].sub_(grads[k][name], alpha=rate / self.scale)
        return loss


class ExpertBlocks(Blocks):
    """``n`` residual blocks whose feed-forward part are ``experts`` experts, of which a router chooses ``k`` for each token."""

    replicated = ("b2", "gamma", "beta", "router")

    def __init__(self, n: int = 2, rows: int = 512, d: int = 256, f: int = 512, experts: int = 8, k: int = 2, devices: int = 4, seed: int = 0):
        torch = self._sizes(n, n * experts, rows, d, f, devices)
        if not 1 <= k <= experts or rows * k % devices:
            raise ValueError("k experts of those there are, and rows times k divisible by the number of devices")
        self.experts, self.k = experts, k
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + 1)
        bf16 = torch.bfloat16

        def weight(out, inner):                                  # feature-sharded tiles of one stack of experts per block
            return [[(torch.randn((experts, out // devices, inner), generator=g, device="cuda") * inner ** -0.5).to(bf16)
                     for _ in range(devices)] for _ in range(n)]

        self.w1, self.w2 = weight(f, d), weight(d, f)
        self.b1 = [[torch.zeros((experts, f // devices), device="cuda") for _ in range(devices)] for _ in range(n)]
        self.b2 = [torch.zeros((experts, d), device="cuda") for _ in range(n)]
        self.gamma, self.beta = [torch.ones(d, device="cuda") for _ in range(n)], [torch.zeros(d, device="cuda") for _ in range(n)]
        self.router = [torch.randn((experts, d), generator=g, device="cuda") * d ** -0.5 for _ in range(n)]
        self.momentum = {"w1": [[torch.zeros_like(t, dtype=torch.float32) for t in w] for w in self.w1],
                         "w2": [[torch.zeros_like(t, dtype=torch.float32) for t in w] for w in self.w2]}

    def own_rows(self, offsets, i: int):
        """Where the experts' rows begin within the rows of device ``i``."""
        share = self.rows * self.k // self.devices
        return (offsets - i * share).clamp(0, share)

    def forward(self, k: int, x: List):
        R, P, d, f, E, devices = self.rows, self.rows * self.k, self.d, self.f, self.experts, range(self.devices)
        norms = [api.layer_norm_forward(x[i], self.gamma[k], self.beta[k]) for i in devices]
        router = self.router[k].to(x[0].dtype)
        logits = self.move([api.linear_forward(y, router) for y, _, _ in norms], (R, E), 0, None)
        routes = [api.route_forward(logits[j], self.k) for j in devices]        # the same on every device
        tokens = self.move([y for y, _, _ in norms], (R, d), 0, 1)
        full = self.move([api.dispatch_forward(tokens[j], routes[j][2]) for j in devices], (P, d), 1, None)
        z = [self.torch.empty((P, f // self.devices), dtype=x[0].dtype, device="cuda") for _ in devices]
        u = [api.experts_forward(full[j], self.w1[k][j], routes[j][3], bias=self.b1[k][j], activation="gelu", pre=z[j]) for j in devices]
        u = self.move(u, (P, f), 1, 0)
        w2 = self.move(self.w2[k], (E, d, f), 1, None)
        begin = [self.own_rows(routes[i][3], i) for i in devices]
        y = self.move([api.experts_forward(u[i], w2[i], begin[i], bias=self.b2[k]) for i in devices], (P, d), 0, 1)
        residual = self.move(x, (R, d), 0, 1)
        out = [api.combine_forward(y[j], routes[j][2], routes[j][0], residual=residual[j]) for j in devices]
        return self.move(out, (R, d), 1, 0), (x, norms, router, logits, routes, full, z, u, w2, begin, y)

    def backward(self, k: int, dy: List, kept):
        x, norms, router, logits, routes, full, z, u, w2, begin, y = kept
        R, P, d, f, E, devices = self.rows, self.rows * self.k, self.d, self.f, self.experts, range(self.devices)
        share = P // self.devices
        # back to the experts' rows; the weights' gradients are sums over the columns, which are spread over the devices
        dy_cols = self.move(dy, (R, d), 0, 1)
        parts = [api.combine_backward(dy_cols[j], y[j], routes[j][2], routes[j][0]) for j in devices]
        dweights = sum(p[1] for p in parts)
        # second product: dw2 of a device's own features needs its columns of the rows' gradient and all of u
        u_full = self.move(u, (P, f), 0, None)
        second = [api.experts_backward(parts[j][0], u_full[j], self.w2[k][j], routes[j][3], need=(False, True, True)) for j in devices]
        dv = self.move([p[0] for p in parts], (P, d), 1, 0)
        du = [api.experts_backward(dv[i], u[i], w2[i], begin[i], need=(True, False, False))[0] for i in devices]
        # first product: the same, with the activation's slope
        du_cols, z_rows, w1 = self.move(du, (P, f), 0, 1), self.move(z, (P, f), 1, 0), self.move(self.w1[k], (E, f, d), 1, None)
        first = [api.experts_backward(du_cols[j], full[j], self.w1[k][j], routes[j][3], z[j], "gelu", need=(False, True, True)) for j in devices]
        drows = [api.experts_backward(du[i], full[i][i * share:(i + 1) * share], w1[i], begin[i], z_rows[i], "gelu", need=(True, False, False))[0]
                 for i in devices]
        drows = self.move(drows, (P, d), 0, 1)
        dn = self.move([api.dispatch_backward(drows[j], routes[j][2]) for j in devices], (R, d), 1, 0)
        # the router
        dlogits = [api.route_backward(dweights, logits[j], routes[j][0], routes[j][1]) for j in devices]
        dlogits = self.move(dlogits, (R, E), None, 0)
        chosen = [api.linear_backward(dlogits[i], norms[i][0], router, need=(True, True, False)) for i in devices]
        back = [api.layer_norm_backward(dn[i] + chosen[i][0], x[i], self.gamma[k], norms[i][1], norms[i][2]) for i in devices]
        dx = [back[i][0] + dy[i] for i in devices]
        return dx, {"w1": [g[1] for g in first], "b1": [g[2] for g in first], "w2": [g[1] for g in second],
                    "b2": self.torch.cat([g[2] for g in second], 1), "gamma": sum(b[1] for b in back), "beta": sum(b[2] for b in back),
                    "router": sum(c[1].float() for c in chosen)}

    def orthogonal(self, name: str, tiles: List[List]) -> List[List]:
        torch, (rows, cols) = self.torch, ((self.f, self.d) if name == "w1" else (self.d, self.f))
        stacks = [torch.cat([tiles[k][j] for k in range(self.n)]) for j in range(self.devices)]
        shape = (self.n * self.experts, rows, cols)
        done = [api.orthogonalize(t, scale=max(1.0, rows / cols) ** 0.5) for t in self.move(stacks, shape, 1, 0)]
        back = self.move(done, shape, 0, 1)
        return [[back[j][k * self.experts:(k + 1) * self.experts] for j in range(self.devices)] for k in range(self.n)]


def main(steps: int = 20, experts: bool = False) -> List[float]:
    import torch

    blocks = ExpertBlocks() if experts else Blocks()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    part = blocks.rows // blocks.devices
    x = [torch.randn((part, blocks.d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(blocks.devices)]
    target = [torch.randn((part, blocks.d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(blocks.devices)]
    losses = []
    for s in range(steps):
        losses.append(float(blocks.step(x, target, clip=1.0 if experts else None)))
        print(f"step {s:3d}  loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    import sys

    main(experts="experts" in sys.argv[1:])
