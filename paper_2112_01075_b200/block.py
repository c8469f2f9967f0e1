"""A training step of sharded residual blocks: the operators on the tiles, redistributions between them.

``python -m paper_2112_01075_b200.block`` trains a few blocks  y = x + gelu(norm(x) w1^T + b1) w2^T + b2  on a mesh of
four virtual devices towards random targets and prints the loss.  Nothing is summed across devices but the layer norm's
weight gradients: wherever a sum over devices would be needed, the operand is brought into the sharding in which the sum
is local.  Types (a: the mesh axis; a device's tile is what the operators see):

    activations      [rows{a}, d]   layer norm, second product with the residual, gradients of the inputs
                     [rows, f{a}]   first product: each device computes its own features
    weights          [f{a}, d], [d{a}, f]: as they are kept, and as their gradients come out
    weight updates   a stack over the blocks, [n, f{a}, d] -> [n{a}, f, d]: whole matrices, orthogonalised where they lie,
                     and back

Every redistribution is planned once and executed on lists of tiles (``api.Plan``).
"""
from __future__ import annotations

from typing import Dict, List

from . import api


class Blocks:
    """``n`` residual blocks of width ``d`` and hidden width ``f`` over ``devices`` virtual devices, bfloat16 weights."""

    def __init__(self, n: int = 4, rows: int = 512, d: int = 256, f: int = 1024, devices: int = 4, seed: int = 0):
        import torch

        if n % devices or rows % devices or d % devices or f % devices:
            raise ValueError("blocks, rows and widths have to be divisible by the number of devices")
        self.torch, self.n, self.rows, self.d, self.f, self.devices = torch, n, rows, d, f, devices
        self.mesh = (devices,)
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
        self._plans: Dict = {}

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

    def step(self, x: List, target: List, rate: float = 0.02, momentum: float = 0.9):
        """One training step; returns the loss before it."""
        loss, grads = self.gradients(x, target)
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
            for name in ("b2", "gamma", "beta"):
                getattr(self, name)[k].sub_(grads[k][name], alpha=rate / self.scale)
        return loss


def main(steps: int = 20) -> List[float]:
    import torch

    blocks = Blocks()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    part = blocks.rows // blocks.devices
    x = [torch.randn((part, blocks.d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(blocks.devices)]
    target = [torch.randn((part, blocks.d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(blocks.devices)]
    losses = []
    for s in range(steps):
        losses.append(float(blocks.step(x, target)))
        print(f"step {s:3d}  loss {losses[-1]:.4f}")
    return losses


if __name__ == "__main__":
    main()
