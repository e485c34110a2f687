"""moe.route as a differentiable operation: the weights' gradient reaches the
logits, as moe.route_backward gives it."""

import numpy as np
import pytest

from oracle import moe as plain
from tests.test_gpu_operators import STEP, U, gpu, host, types  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cfg", [dict(scores="softmax"), dict(scores="softmax", renormalise=False), dict(scores="sigmoid", scale=2.5),
                                 dict(scores="sigmoid", groups=4, groups_kept=2, group_best=2)],
                         ids=lambda c: "-".join(str(v) for v in c.values()))
@pytest.mark.parametrize("pad", [0, 3])
def test_gradient_of_the_logits(gpu, cfg, kind, pad):  # noqa: F811
    torch, moe = gpu
    r = moe.Router(32, 4, **cfg)
    g = torch.Generator(device="cuda").manual_seed(6)
    data = torch.randn((57, 32 + pad), generator=g, device="cuda").to(types(torch)[kind])
    data[3] = -float("inf")
    bias = torch.linspace(-0.1, 0.1, 32, device="cuda")
    leaf = data.clone().requires_grad_()
    dw = torch.randn((57, 4), generator=g, device="cuda")
    e, w = moe.route(r, leaf[:, :32], bias)
    assert w.requires_grad and not e.requires_grad
    plain_e, plain_w = moe.route(r, data[:, :32], bias)
    assert torch.equal(e, plain_e) and torch.equal(w.detach(), plain_w) and not plain_w.requires_grad
    (w * dw).sum().backward()
    want = moe.route_backward(r, data[:, :32], e, dw)
    assert leaf.grad.dtype == data.dtype and torch.equal(leaf.grad[:, :32], want)
    assert (leaf.grad[:, 32:] == 0).all() and (leaf.grad[3] == 0).all()
    exact = plain.route_backward(r, host(data[:, :32]), e.cpu().numpy(), host(dw))
    total = np.abs(host(dw)).sum(1, keepdims=True) * r.scale
    assert (np.abs(host(want) - exact) <= STEP[kind] * np.abs(exact) + 2.0 ** -24 + 200 * U * total).all()


def test_gradients_that_are_not_contiguous(gpu):  # noqa: F811
    """sum() hands back one value for all weights, a product in 64 bits is
    cast: the gradient is that of ordinary ones."""
    torch, moe = gpu
    r = moe.Router(16, 3, "sigmoid", False)
    x = torch.randn((9, 16), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    leaf = x.clone().requires_grad_()
    e, w = moe.route(r, leaf)
    (g,) = torch.autograd.grad(w.sum(), leaf, retain_graph=True)
    assert torch.equal(g, moe.route_backward(r, x, e, torch.ones((9, 3), device="cuda")))
    (g,) = torch.autograd.grad((w.double().t() * 2).sum(), leaf)
    assert torch.equal(g, moe.route_backward(r, x, e, torch.full((9, 3), 2.0, device="cuda")))


def test_without_gradients(gpu):  # noqa: F811
    torch, moe = gpu
    r = moe.Router(16, 3)
    leaf = torch.randn((9, 16), device="cuda").requires_grad_()
    with torch.no_grad():
        assert not moe.route(r, leaf)[1].requires_grad
    with torch.inference_mode():
        assert not moe.route(r, leaf)[1].requires_grad
    with pytest.raises(ValueError):       # the checks are the same
        moe.route(r, leaf[:, :8])


def test_second_derivatives_are_refused(gpu):  # noqa: F811
    torch, moe = gpu
    leaf = torch.randn((9, 16), device="cuda").requires_grad_()
    (g,) = torch.autograd.grad((moe.route(moe.Router(16, 3, "sigmoid"), leaf)[1] ** 2).sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
