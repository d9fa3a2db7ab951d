"""ctypes binding of `include/dhq_groups.h`: products with 4-bit weights, activation checkpoints in 8 bits.

Names and meaning follow the header.  Matrices are 2-d torch CUDA tensors on the current device whose rows may be strided
(last dimension contiguous); results go to tensors that the caller passes.  `stream` is a torch stream of the current
device (default: its current stream).  Storage for `rows` x K values in groups of G, Kp = `padded_columns(K, G)`:
4-bit codes uint8 [N][Kp / 2] with scales bfloat16 [N][Kp / G]; checkpoints int8 [T][Kp] with exponents uint8 [T][Kp / G];
these four are contiguous.
"""
from __future__ import annotations

import ctypes
from functools import lru_cache

import torch

from .binding import DHQ_ACT_SINE, DHQ_ROT_NONE, DhqError, _current_device, _raw_stream, load_library

DHQ_ACT_NONE = 2
DHQ_ACT_SILU = 3
DHQ_ACT_GELU = 4
DHQ_F32, DHQ_BF16, DHQ_F16 = 0, 1, 2

_TYPES = {torch.float32: DHQ_F32, torch.bfloat16: DHQ_BF16, torch.float16: DHQ_F16}
_fn = {}


def _functions():
    """The library's functions, looked up and declared once (calls of a few microseconds of device time go through here)."""
    if not _fn:
        L = load_library()
        vp, i, n, f = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
        kinds = {
            "dhq_w4_pack": [vp, i, n, n, n, i, i, vp, vp, vp],
            "dhq_w4_linear_workspace": [n, n, n, i, i, i, ctypes.POINTER(n)],
            "dhq_w4_linear": [vp, vp, n, n, i, i, vp, i, n, n, vp, vp, n, vp, n, vp],
            "dhq_checkpoint_save": [vp, i, n, n, n, i, i, i, f, f, vp, vp, vp, n, vp],
            "dhq_checkpoint_act_grad": [vp, vp, n, n, i, i, i, f, f, vp, i, n, vp, n, vp],
            "dhq_checkpoint_weight_grad_workspace": [n, n, n, i, i, i, vp, n, i, ctypes.POINTER(n)],
            "dhq_checkpoint_weight_grad": [vp, vp, n, n, i, i, vp, i, n, n, vp, i, n, vp, n, vp],
        }
        for name, kind in kinds.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = kind, i
        _fn.update({name: getattr(L, name) for name in kinds})
    return _fn


def padded_columns(k: int, group: int) -> int:
    """Columns of a row of k values in whole groups."""
    return -(-k // group) * group


# The calls below take a few microseconds of device time for few rows, so each looks at a tensor's properties once (some 0.1 us each) and leaves
# the finding of what is wrong to the functions that raise.

def _bad_matrix(t, what, dtype=None, shape=None, device=None):
    """Raises what a matrix argument is refused for; returns if there is nothing."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2):
        raise TypeError(f"{what}: expected a CUDA tensor of two dimensions")
    if t.dtype not in _TYPES if dtype is None else t.dtype != dtype:
        raise TypeError(f"{what}: expected dtype {dtype or 'float32, bfloat16 or float16'}")
    if t.size(1) > 1 and t.stride(1) != 1:
        raise TypeError(f"{what}: the last dimension has to be contiguous")
    if shape is not None and tuple(t.shape) != shape:
        raise ValueError(f"{what}: expected shape {shape}, got {tuple(t.shape)}")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{what}: on another device than the other arguments")


def _matrix(t, what):
    """(rows, columns, leading dimension, device, address) of a matrix of any of the types."""
    try:
        (rows, columns), strides, device = t.shape, t.stride(), t.get_device()
    except (AttributeError, ValueError):
        rows = -1
    if rows < 0 or device < 0 or t.dtype not in _TYPES or (columns > 1 and strides[1] != 1):
        _bad_matrix(t, what)
    # (a tensor of one row may carry any stride there)
    return rows, columns, strides[0] if rows > 1 else columns, device, t.data_ptr()


def _result(t, what, dtype, shape, device):
    """(leading dimension, address) of a matrix of this type, shape and device."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _bad_matrix(t, what, dtype, shape, device)
    strides = t.stride()
    if shape[1] > 1 and strides[1] != 1:
        _bad_matrix(t, what, dtype, shape, device)
    return strides[0] if shape[0] > 1 else shape[1], t.data_ptr()


def _store(t, what, dtype, shape, device):
    """Address of a tensor of the library's own storage format."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
            raise TypeError(f"{what}: expected a contiguous CUDA tensor of dtype {dtype}")
        if tuple(t.shape) != shape:
            raise ValueError(f"{what}: expected shape {shape}, got {tuple(t.shape)}")
        raise ValueError(f"{what}: on another device than the other arguments")
    return t.data_ptr()


def _stream_of(stream, device):
    if device != _current_device():
        raise ValueError(f"tensors are on cuda:{device}, which is not the current device")
    if stream is None:
        return _raw_stream(device)
    if stream.device_index != device:
        raise ValueError(f"the stream belongs to another device than the tensors (cuda:{device})")
    return stream.cuda_stream


def _padded(k, group):
    if group not in (32, 64, 128):
        raise DhqError(2, "group (32, 64 or 128)")
    return -(-k // group) * group


def _need(name, *sizes):
    need = ctypes.c_int64()
    code = _functions()[name](*sizes, ctypes.byref(need))
    if code:
        raise DhqError(code, name)
    return need.value


def _workspace(workspace, need, device, stream):
    """(address, bytes, tensor to keep) of the caller's workspace, or of one for this call."""
    if workspace is None:
        if not need:
            return None, 0, None
        if stream is None:
            workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        else:   # allocated on the stream that uses it, so that its memory is given to nobody else before this call's work is done
            with torch.cuda.stream(stream):
                workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
    elif not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous() and workspace.dtype == torch.uint8
              and workspace.get_device() == device):
        raise TypeError("workspace: expected a contiguous CUDA tensor of dtype uint8 on the other arguments' device")
    return workspace.data_ptr(), workspace.numel(), workspace


def dhq_w4_pack(weight, codes, scales, group=128, rotation=DHQ_ROT_NONE, stream=None):
    """weight [N][K] -> codes, scales."""
    n, k, lead, device, address = _matrix(weight, "weight")
    padded = _padded(k, group)
    code = _functions()["dhq_w4_pack"](
        address, _TYPES[weight.dtype], n, k, lead, group, rotation, _store(codes, "codes", torch.uint8, (n, padded // 2), device),
        _store(scales, "scales", torch.bfloat16, (n, padded // group), device), _stream_of(stream, device))
    if code:
        raise DhqError(code, "dhq_w4_pack")


@lru_cache(maxsize=1024)   # (sizes and types alone decide; a call of a few microseconds of device time asks each time)
def _linear_need(*sizes):
    return _need("dhq_w4_linear_workspace", *sizes)


def dhq_w4_linear_workspace(t, n, k, dtype, group=128, rotation=DHQ_ROT_NONE) -> int:
    """Bytes that dhq_w4_linear needs beside its arguments."""
    return _linear_need(t, n, k, group, rotation, _TYPES[dtype])


def dhq_w4_linear(codes, scales, x, out, bias=None, group=128, rotation=DHQ_ROT_NONE, workspace=None, stream=None):
    """out[t][n] = x[t] . W[n] (+ bias[n]); x [T][K], out [T][N] and bias [N] of one dtype.  workspace: a uint8 tensor of
    dhq_w4_linear_workspace bytes, else one is taken from torch's allocator for this call where one is needed."""
    t, k, lead, device, address = _matrix(x, "x")
    dtype = x.dtype
    n = out.shape[1] if isinstance(out, torch.Tensor) and out.dim() == 2 else -1
    out_lead, out_address = _result(out, "out", dtype, (t, n), device)
    padded = _padded(k, group)
    raw = _stream_of(stream, device)
    where, size, _keep = _workspace(workspace, _linear_need(t, n, k, group, rotation, _TYPES[dtype]), device, stream)
    code = _functions()["dhq_w4_linear"](
        _store(codes, "codes", torch.uint8, (n, padded // 2), device), _store(scales, "scales", torch.bfloat16, (n, padded // group), device), n, k,
        group, rotation, address, _TYPES[dtype], t, lead, None if bias is None else _store(bias, "bias", dtype, (n,), device),
        out_address, out_lead, where, size, raw)
    if code:
        raise DhqError(code, "dhq_w4_linear")


def dhq_checkpoint_save(x, codes, exponents, out=None, activation=DHQ_ACT_NONE, omega0=30.0, act_s0=0.0, group=128,
                        rotation=DHQ_ROT_NONE, stream=None):
    """Checkpoint of x [T][K], and out = act(x) unless the activation is DHQ_ACT_NONE (out may be x).  codes and exponents None: out alone."""
    t, k, lead, device, address = _matrix(x, "x")
    padded = _padded(k, group)
    out_lead, out_address = 0, None
    if out is not None:
        out_lead, out_address = _result(out, "out", x.dtype, (t, k), device)
    elif activation != DHQ_ACT_NONE:
        raise TypeError("out: the activation's result needs a tensor")
    kept = None, None
    if codes is not None or exponents is not None:
        kept = _store(codes, "codes", torch.int8, (t, padded), device), _store(exponents, "exponents", torch.uint8, (t, padded // group), device)
    code = _functions()["dhq_checkpoint_save"](
        address, _TYPES[x.dtype], t, k, lead, group, rotation, activation, omega0, act_s0, *kept, out_address, out_lead, _stream_of(stream, device))
    if code:
        raise DhqError(code, "dhq_checkpoint_save")


def dhq_checkpoint_act_grad(codes, exponents, grad_out, grad_in, activation=DHQ_ACT_SINE, omega0=30.0, act_s0=0.0, group=128,
                            rotation=DHQ_ROT_NONE, stream=None):
    """grad_in = grad_out act'(x^), x^ being what the checkpoint stands for (grad_in may be grad_out)."""
    t, k, lead, device, address = _matrix(grad_out, "grad_out")
    padded = _padded(k, group)
    in_lead, in_address = _result(grad_in, "grad_in", grad_out.dtype, (t, k), device)
    code = _functions()["dhq_checkpoint_act_grad"](
        _store(codes, "codes", torch.int8, (t, padded), device), _store(exponents, "exponents", torch.uint8, (t, padded // group), device), t, k, group,
        rotation, activation, omega0, act_s0, address, _TYPES[grad_out.dtype], lead, in_address, in_lead, _stream_of(stream, device))
    if code:
        raise DhqError(code, "dhq_checkpoint_act_grad")


def dhq_checkpoint_weight_grad_workspace(grad_out, grad_weight, group=128, rotation=DHQ_ROT_NONE) -> int:
    """Bytes that dhq_checkpoint_weight_grad needs beside these arguments."""
    t, n, lead, _, address = _matrix(grad_out, "grad_out")
    return _need("dhq_checkpoint_weight_grad_workspace", t, n, grad_weight.size(1), group, rotation, _TYPES[grad_out.dtype], address, lead,
                 _TYPES[grad_weight.dtype])


def dhq_checkpoint_weight_grad(codes, exponents, grad_out, grad_weight, group=128, rotation=DHQ_ROT_NONE, workspace=None, stream=None):
    """grad_weight [N][K] = grad_out [T][N]^T x^ [T][K]; grad_weight fp32 or of grad_out's dtype.  workspace: a uint8 tensor of
    dhq_checkpoint_weight_grad_workspace bytes, else one is taken from torch's allocator for this call."""
    t, n, lead, device, address = _matrix(grad_out, "grad_out")
    kind = _TYPES[grad_out.dtype]
    k = grad_weight.shape[1] if isinstance(grad_weight, torch.Tensor) and grad_weight.dim() == 2 else -1
    out_type = torch.float32 if isinstance(grad_weight, torch.Tensor) and grad_weight.dtype is torch.float32 else grad_out.dtype
    out_lead, out_address = _result(grad_weight, "grad_weight", out_type, (n, k), device)
    padded = _padded(k, group)
    raw = _stream_of(stream, device)
    need = _need("dhq_checkpoint_weight_grad_workspace", t, n, k, group, rotation, kind, address, lead, _TYPES[out_type])
    where, size, _keep = _workspace(workspace, need, device, stream)
    code = _functions()["dhq_checkpoint_weight_grad"](
        _store(codes, "codes", torch.int8, (t, padded), device), _store(exponents, "exponents", torch.uint8, (t, padded // group), device), t, k, group,
        rotation, address, kind, n, lead, out_address, _TYPES[out_type], out_lead, where, size, raw)
    if code:
        raise DhqError(code, "dhq_checkpoint_weight_grad")
