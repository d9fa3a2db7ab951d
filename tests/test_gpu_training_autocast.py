"""Layers with checkpoints under torch.autocast."""
import pytest
import torch

from tests import groups_ref as ref
import paper_2508_13478_b200 as dhq

pytestmark = pytest.mark.gpu


def normal(*shape, seed=0, scale=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda() * scale


@pytest.mark.parametrize("kept", [torch.float32, torch.bfloat16, torch.float16])   # type of the layer's input
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rotation", [dhq.DHQ_ROT_NONE, dhq.DHQ_ROT_INPUT])
def test_linear_under_autocast(kept, dtype, rotation):
    x = normal(3, 70, 100).to(kept).requires_grad_()
    w = normal(50, 100, seed=1, scale=0.1).requires_grad_()
    b = normal(50, seed=2).requires_grad_()
    with torch.autocast("cuda", dtype):
        y = dhq.checkpointed_linear(x, w, b, 64, rotation)
    assert y.dtype == dtype and torch.equal(y, torch.nn.functional.linear(x.to(dtype), w.to(dtype), b.to(dtype)))
    dy = normal(3, 70, 50, seed=3).to(dtype)
    y.backward(dy)     # (outside of autocast, as torch wants it)
    dy2 = dy.reshape(-1, 50)
    assert x.grad.dtype == kept and w.grad.dtype == b.grad.dtype == torch.float32
    assert torch.equal(x.grad, (dy2 @ w.detach().to(dtype)).reshape(x.shape).to(kept))
    # the gradients of fp32 weights and biases are not rounded to the gradient's type on their way
    want = dy2.double().sum(0)
    assert ((b.grad.double() - want).abs() <= 210 * 2.0 ** -24 * dy2.double().abs().sum(0)).all()
    rotate = rotation == dhq.DHQ_ROT_INPUT
    codes, stored = ref.checkpoint8(x.detach().reshape(-1, 100), 64, rotate)
    z, plain = ref.restored64(codes, stored, 64, rotate, 100), ref.restored64(codes, stored, 64, False, 128)
    spread = ((dy2.double() ** 2).T @ plain ** 2).reshape(50, -1, 64).mean(-1, keepdim=True).expand(-1, -1, 64).flatten(1)[:, :100].sqrt()
    if not rotate:
        spread = ((dy2.double() ** 2).T @ plain[:, :100] ** 2).sqrt()
    ref.assert_sums(w.grad, dy2.double().T @ z, spread, 210 // 16 + 60 + 64)


@pytest.mark.parametrize("weights", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_weights_of_either_16_bit_type_under_autocast(weights, dtype):
    x, w = normal(90, 64).requires_grad_(), normal(20, 64, seed=1, scale=0.1).to(weights).requires_grad_()
    with torch.autocast("cuda", dtype):
        y = dhq.checkpointed_linear(x, w)
    dy = normal(90, 20, seed=3).to(dtype)
    y.backward(dy)
    assert torch.equal(x.grad, (dy @ w.detach().to(dtype)).float())
    codes, stored = ref.checkpoint8(x.detach(), 64, True)
    want, plain = dy.double().T @ ref.restored64(codes, stored, 64, True, 64), ref.restored64(codes, stored, 64, False, 64)
    spread = ((dy.double() ** 2).T @ plain ** 2).mean(-1, keepdim=True).expand(-1, 64).sqrt()
    ref.assert_sums(w.grad, want, spread, 90 // 16 + 60 + 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_step_of_a_network_under_autocast(dtype):
    x, target = normal(333, 96), normal(333, 33, seed=2)
    w = [normal(128, 96, seed=3).mul(0.1).requires_grad_(), normal(33, 128, seed=4).mul(0.1).requires_grad_()]

    def gradients(linear, act):
        with torch.autocast("cuda", dtype):
            out = linear(act(linear(x, w[0])), w[1])
            return torch.autograd.grad(((out - target) ** 2).mean(), w)   # (a backward pass within autocast is allowed, too)

    got = gradients(dhq.checkpointed_linear, lambda z: dhq.checkpointed_activation(z, dhq.DHQ_ACT_SILU))
    like = gradients(torch.nn.functional.linear, torch.nn.functional.silu)
    for a, b in zip(got, like):   # checkpoints are off by up to 1 / 127 of a group's largest value, independent from row to row
        assert a.dtype == torch.float32 and torch.nn.functional.cosine_similarity(a.flatten(), b.flatten(), dim=0).item() > 0.99
