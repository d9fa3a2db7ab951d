"""Layers with checkpoints where no backward pass can come, and the call below them without a checkpoint."""
import ctypes as C

import pytest
import torch

import paper_2508_13478_b200 as dhq
from paper_2508_13478_b200 import training


def normal(*shape, seed=0, scale=1.0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).cuda() * scale


def no_storage(*_):
    raise AssertionError("a checkpoint that nothing will read")


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["no_grad", "inference_mode", "no gradient asked for"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_nothing_is_kept_where_no_backward_pass_can_come(monkeypatch, mode, dtype):
    x, w, b = normal(7, 11, 95).to(dtype), normal(50, 95, seed=1).to(dtype), normal(50, seed=2).to(dtype)
    wide = normal(77, 96).to(dtype)
    acts = {dhq.DHQ_ACT_SINE: 0.1, dhq.DHQ_ACT_GABOR: 0.05, dhq.DHQ_ACT_SILU: 2.0, dhq.DHQ_ACT_GELU: 2.0}

    def run(grad):
        ws = [w, b] if mode == "no gradient asked for" else [w.requires_grad_(), b.requires_grad_()]
        outs = [dhq.checkpointed_linear(x, *ws)]
        for act, scale in acts.items():
            for v in (x, wide, wide[:, :32]):
                z = (v * scale).requires_grad_(grad or mode != "no gradient asked for")
                outs.append(dhq.checkpointed_activation(z, act, 30.0, 10.0, 32))
        return outs

    want = [y.detach() for y in run(True)]
    w, b = w.detach(), b.detach()
    monkeypatch.setattr(training, "_storage", no_storage)
    if mode == "no gradient asked for":
        got = run(False)
    else:
        with getattr(torch, mode)():
            got = run(False)
    assert all(torch.equal(a, y) and not y.requires_grad for a, y in zip(want, got))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("act", [dhq.DHQ_ACT_SINE, dhq.DHQ_ACT_GABOR, dhq.DHQ_ACT_SILU, dhq.DHQ_ACT_GELU])
def test_the_activation_alone_has_the_same_bits(dtype, act):
    for t, k, lead in ((1, 1, 1), (5, 127, 127), (333, 70, 72), (9, 1000, 1008), (4000, 512, 512), (3000, 700, 701)):
        form = dict(activation=act, omega0=30.0, act_s0=10.0, group=64, rotation=dhq.DHQ_ROT_INPUT)
        x = normal(t, lead, seed=t, scale=0.1).to(dtype)[:, :k]
        codes, exponents = training._storage(t, k, 64, x.device)
        want = torch.empty(t, k, dtype=dtype, device="cuda")
        dhq.dhq_checkpoint_save(x, codes, exponents, out=want, **form)
        around = torch.full((t, lead + 3), 7.0, dtype=dtype, device="cuda")
        dhq.dhq_checkpoint_save(x, None, None, out=around[:, :k], **form)
        assert torch.equal(around[:, :k], want) and (around[:, k:] == 7).all()
        dhq.dhq_checkpoint_save(x, None, None, out=x, **form)   # in place
        assert torch.equal(x, want)


@pytest.mark.gpu
def test_half_a_checkpoint_is_refused():
    x = normal(4, 64)
    codes, exponents = training._storage(4, 64, 32, x.device)
    form = dict(activation=dhq.DHQ_ACT_SILU, group=32, out=torch.empty_like(x))
    for kept in ((codes, None), (None, exponents)):
        with pytest.raises(TypeError):
            dhq.dhq_checkpoint_save(x, *kept, **form)
    with pytest.raises(dhq.DhqError):
        dhq.dhq_checkpoint_save(x, None, None, activation=dhq.DHQ_ACT_NONE, group=32)


def test_half_a_checkpoint_is_refused_by_the_library():
    from paper_2508_13478_b200 import build
    L = C.CDLL(build.build())
    vp, i, n, f = C.c_void_p, C.c_int, C.c_int64, C.c_float
    L.dhq_checkpoint_save.argtypes = [vp, i, n, n, n, i, i, i, f, f, vp, vp, vp, n, vp]
    P = 1 << 20   # stands for a device address; nothing reads it
    for act, codes, exponents, y in ((3, P, None, P), (3, None, P, P), (2, None, None, None), (2, None, P, None), (3, None, None, None)):
        assert L.dhq_checkpoint_save(P, 0, 2, 100, 100, 64, 0, act, 0.0, 0.0, codes, exponents, y, 100, None) == 1


def test_linear_layer_without_gradients_is_the_product(monkeypatch):
    monkeypatch.setattr(training, "_storage", no_storage)
    x, w, b = torch.randn(2, 5, 8), torch.randn(3, 8, requires_grad=True), torch.randn(3, requires_grad=True)
    with torch.no_grad():
        assert torch.allclose(dhq.checkpointed_linear(x, w, b), torch.nn.functional.linear(x, w, b), atol=1e-5)
        assert dhq.checkpointed_linear(x[:, :0], w).shape == (2, 0, 3)
