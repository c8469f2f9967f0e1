"""The sharded residual blocks: gradients against autograd on the global arrays, and a training run."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def whole(tiles):
    return torch.cat(tiles).float().requires_grad_()


def test_gradients_match_autograd_on_the_global_arrays():
    """bfloat16 keeps 8 bits: a tensor's rounding is 2^-9 of it on average, about a dozen tensors lie between a weight and
    the loss and each adds its own, so gradients agree to sqrt(12) 2^-9 = 0.7 %; four times that is allowed."""
    from paper_2112_01075_b200.block import Blocks
    b = Blocks(n=2, rows=128, d=96, f=160, devices=2, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = [torch.randn((64, 96), generator=g, device="cuda").bfloat16() for _ in range(2)]
    target = [torch.randn((64, 96), generator=g, device="cuda").bfloat16() for _ in range(2)]
    for k in range(2):                                       # nothing at its neutral value
        for t in b.b1[k] + [b.b2[k], b.gamma[k], b.beta[k]]:
            t.add_(torch.randn(t.shape, generator=g, device="cuda") * 0.1)
    loss, grads = b.gradients(x, target)

    params, h = [], torch.cat(x).float()
    for k in range(2):
        p = dict(w1=whole(b.w1[k]), w2=whole(b.w2[k]), b1=whole(b.b1[k]), b2=whole([b.b2[k]]), gamma=whole([b.gamma[k]]), beta=whole([b.beta[k]]))
        params.append(p)
        n = (h - h.mean(1, keepdim=True)) * torch.rsqrt(h.var(1, unbiased=False, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
        u = n @ p["w1"].T + p["b1"]
        h = h + (u * 0.5 * torch.special.erfc(-u / 2 ** 0.5)) @ p["w2"].T + p["b2"]
    want = ((h - torch.cat(target).float()) ** 2).mean()
    want.backward()
    assert abs(float(loss - want)) < 1e-2 * float(want)
    for k in range(2):
        for name, p in params[k].items():
            got = grads[k][name]
            got = (torch.cat(got) if isinstance(got, list) else got).float() / b.scale
            off = float((got - p.grad).norm() / p.grad.norm())
            assert off < 0.028, (k, name, off)


def test_a_few_steps_lower_the_loss():
    from paper_2112_01075_b200 import api, block
    before = api.redist_product_timeouts()
    losses = block.main(12)
    assert losses[-1] < 0.7 * losses[0] and api.redist_product_timeouts() == before and api.redist_bulk_timeouts() == 0
