"""Layers whose backward pass works from 8-bit checkpoints: autograd functions around `groups`.

Between forward and backward pass a linear layer keeps its input, and an activation what it was applied to, as 8-bit codes with a power
of two per group of consecutive features (1 + 1 / group bytes a value in place of 4 or 2).  Gradients with respect to inputs of a
linear layer need its weights only and are exact; weight gradients and slopes of activations see the checkpoint's values.

Under torch.autocast a linear layer multiplies in autocast's type, forward and backward, as torch's own does; it keeps its input as it came, and
the gradient of fp32 weights is summed and written in fp32.

Where no backward pass can follow (gradients are off, or none is asked for) nothing is kept.

A forward and backward pass may be captured into a CUDA graph in torch's way: warmed up on a side stream, with no eager graph of the same
leaves alive when the capture begins (torch's gradient accumulation would wait for a stream that is not being captured).
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from .binding import DHQ_ACT_GABOR, DHQ_ACT_SINE, DHQ_ROT_INPUT
from .groups import (DHQ_ACT_NONE, dhq_checkpoint_act_grad, dhq_checkpoint_save, dhq_checkpoint_weight_grad, padded_columns)

__all__ = ["checkpointed_linear", "checkpointed_activation", "DHQ_ACT_SINE", "DHQ_ACT_GABOR"]


def _storage(rows, k, group, device):
    padded = padded_columns(k, group)
    return (torch.empty(rows, padded, dtype=torch.int8, device=device),
            torch.empty(rows, padded // group, dtype=torch.uint8, device=device))


def _rows(t):
    """t as a matrix whose last dimension is contiguous and whose rows do not overlap."""
    t = t.reshape(-1, t.shape[-1])
    fits = (t.shape[1] == 1 or t.stride(1) == 1) and (t.shape[0] == 1 or t.stride(0) >= t.shape[1])
    return t if fits else t.clone(memory_format=torch.contiguous_format)


def _product(x, x2, weight, bias):
    y = x2 @ weight.t() if bias is None else torch.addmm(bias, x2, weight.t())
    return y.reshape(*x.shape[:-1], weight.shape[0])


class _Linear(torch.autograd.Function):
    @staticmethod
    @torch.amp.custom_fwd(device_type="cuda")
    def forward(ctx, x, weight, bias, group, rotation):
        x2 = _rows(x)
        ctx.form, ctx.shape = (group, rotation), x.shape
        codes = exponents = None
        if ctx.needs_input_grad[1]:
            codes, exponents = _storage(x2.shape[0], x2.shape[1], group, x.device)
            dhq_checkpoint_save(x2, codes, exponents, activation=DHQ_ACT_NONE, group=group, rotation=rotation)
        ctx.save_for_backward(weight, codes, exponents)
        return _product(x, x2, weight, bias)

    @staticmethod
    @once_differentiable
    @torch.amp.custom_bwd(device_type="cuda")   # (the products below take the types that the forward pass took)
    def backward(ctx, dy):
        weight, codes, exponents = ctx.saved_tensors
        group, rotation = ctx.form
        dy2 = _rows(dy)
        dx = (dy2 @ weight).reshape(ctx.shape) if ctx.needs_input_grad[0] else None
        dw = None
        if ctx.needs_input_grad[1]:
            # (16-bit weights under autocast of the other 16-bit type: fp32, which autograd rounds to theirs)
            dw = torch.empty(weight.shape, dtype=weight.dtype if weight.dtype == dy.dtype else torch.float32, device=weight.device)
            dhq_checkpoint_weight_grad(codes, exponents, dy2, dw, group=group, rotation=rotation)
        db = dy2.sum(0) if ctx.needs_input_grad[2] else None
        return dx, dw, db, None, None


def _activate(z, keep, form):
    """act(z), and the checkpoint's codes and exponents (None unless they are kept)."""
    z2 = _rows(z)
    codes, exponents = _storage(z2.shape[0], z2.shape[1], form["group"], z.device) if keep else (None, None)
    y = torch.empty(z2.shape, dtype=z.dtype, device=z.device)
    dhq_checkpoint_save(z2, codes, exponents, out=y, **form)
    return y.reshape(z.shape), codes, exponents


class _Activation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, form):
        y, codes, exponents = _activate(z, True, form)
        ctx.save_for_backward(codes, exponents)
        ctx.form = form
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        codes, exponents = ctx.saved_tensors
        dy2 = _rows(dy)
        dz = torch.empty(dy2.shape, dtype=dy.dtype, device=dy.device)
        dhq_checkpoint_act_grad(codes, exponents, dy2, dz, **ctx.form)
        return dz.reshape(dy.shape), None


def checkpointed_linear(x, weight, bias=None, group=64, rotation=DHQ_ROT_INPUT):
    """x weight^T + bias (fp32, bf16 or fp16 CUDA tensors, of one dtype unless autocast is on; x [..., K]), keeping x as an 8-bit checkpoint for the weight's gradient."""
    if not torch.is_grad_enabled():   # (within a function of autograd it always is off)
        return _product(x, _rows(x), weight, bias)
    return _Linear.apply(x, weight, bias, group, rotation)


def checkpointed_activation(z, activation=DHQ_ACT_SINE, omega0=30.0, act_s0=0.0, group=64, rotation=DHQ_ROT_INPUT):
    """act(z), keeping z as an 8-bit checkpoint for the slope; activations as for dhq_checkpoint_save, but DHQ_ACT_NONE."""
    form = dict(activation=activation, omega0=omega0, act_s0=act_s0, group=group, rotation=rotation)
    if not (torch.is_grad_enabled() and z.requires_grad):
        return _activate(z, False, form)[0]
    return _Activation.apply(z, form)
