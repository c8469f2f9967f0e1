"""The sharded residual blocks with experts: gradients against autograd on the global arrays, clipped gradients, and a step."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def make(n=2, rows=128, d=96, f=160, experts=6, k=2, devices=2, seed=3):
    from paper_2112_01075_b200.block import ExpertBlocks
    b = ExpertBlocks(n, rows, d, f, experts, k, devices, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = [torch.randn((rows // devices, d), generator=g, device="cuda").bfloat16() for _ in range(devices)]
    target = [torch.randn((rows // devices, d), generator=g, device="cuda").bfloat16() for _ in range(devices)]
    for i in range(n):                                       # nothing at its neutral value
        for t in b.b1[i] + [b.b2[i], b.gamma[i], b.beta[i]]:
            t.add_(torch.randn(t.shape, generator=g, device="cuda") * 0.1)
    return b, x, target


def test_gradients_match_autograd_on_the_global_arrays():
    """bfloat16 tensors between the operators: a tensor's rounding is 2^-9 of it on average, about sixteen tensors lie between a
    weight and the loss and each adds its own: sqrt(16) 2^-9 = 0.8 %; four times that is allowed.  The choice of experts is taken
    from the blocks: a choice that rounding decides otherwise would be another function."""
    b, x, target = make()
    choices = []
    real = type(b).forward

    def forward(self, k, v):
        out, kept = real(self, k, v)
        choices.append(kept[4][0][1].long())
        return out, kept

    type(b).forward = forward
    try:
        loss, grads = b.gradients(x, target)
    finally:
        type(b).forward = real
    leaf = lambda t: t.float().requires_grad_()                                          # noqa: E731
    params, h = [], torch.cat(x).float()
    for i in range(2):
        p = dict(w1=leaf(torch.cat(b.w1[i], 1)), w2=leaf(torch.cat(b.w2[i], 1)), b1=leaf(torch.cat(b.b1[i], 1)), b2=leaf(b.b2[i]), gamma=leaf(b.gamma[i]),
                 beta=leaf(b.beta[i]), router=leaf(b.router[i]))
        p = {name: t.detach().requires_grad_() for name, t in p.items()}
        params.append(p)
        n = (h - h.mean(1, keepdim=True)) * torch.rsqrt(h.var(1, unbiased=False, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
        weights = torch.softmax((n @ p["router"].T).gather(1, choices[i]), 1)
        y = h
        for s in range(2):
            e = choices[i][:, s]
            u = torch.einsum("td,tfd->tf", n, p["w1"][e]) + p["b1"][e]
            u = u * 0.5 * torch.special.erfc(-u / 2 ** 0.5)
            y = y + weights[:, s:s + 1] * (torch.einsum("tf,tdf->td", u, p["w2"][e]) + p["b2"][e])
        h = y
    want = ((h - torch.cat(target).float()) ** 2).mean()
    want.backward()
    assert abs(float(loss.detach() - want.detach())) < 1e-2 * float(want.detach())
    for i in range(2):
        for name, p in params[i].items():
            got = grads[i][name]
            got = (torch.cat(got, 1) if isinstance(got, list) else got).float() / b.scale
            off = float((got - p.grad).norm() / p.grad.norm())
            assert off < 0.032, (i, name, off)


def test_clipped_gradients():
    b, x, target = make()
    _, grads = b.gradients(x, target)
    every = [t for g in grads for v in g.values() for t in (v if isinstance(v, list) else [v])]
    norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in every)) / b.scale
    got = float(b.clip(grads, norm / 8))
    assert abs(got - norm) < 1e-5 * norm
    after = math.sqrt(sum(float((t.double() ** 2).sum()) for t in every)) / b.scale
    assert abs(after - norm / 8) < 2.0 ** -8 * norm / 8


@pytest.mark.parametrize("devices,n,experts,k", [(2, 1, 4, 1), (4, 2, 8, 2), (4, 1, 4, 3)])
def test_steps_run(devices, n, experts, k):
    from paper_2112_01075_b200 import api
    before = api.redist_product_timeouts()
    b, x, target = make(n, 64, 64, 128, experts, k, devices)
    for clip in (None, 0.1):
        assert math.isfinite(float(b.step(x, target, clip=clip)))
    assert all(bool(torch.isfinite(t).all()) for w in (b.w1, b.w2, b.b1) for tiles in w for t in tiles)
    assert api.redist_product_timeouts() == before and api.redist_bulk_timeouts() == 0
