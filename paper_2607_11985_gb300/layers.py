"""Classical operators of a hybrid model, for torch CUDA tensors.

What stands around a ``Circuit`` inside a network, in the library's kernels:

  layer_norm   y = (x - mean) / sqrt(var + eps) * weight + bias over the last axis
  linear       y = act(x weight^T + bias) + residual: features to a circuit's
               angles, expectations back to features, ordinary projections
  gated        h = act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up)

Each has three forms: ``linear_forward`` and ``linear_backward`` are the two
launches of a training step (or inference with ``save=False``), ``linear`` the
same under autograd.  x may have any leading axes; rows may be strided (other
layouts are copied).  Types: float32, bfloat16 and float16, sums and
statistics in float; see include/vqc.h for the formulas and roundings.  Torch
supplies device memory and the current stream only.
"""
from __future__ import annotations

import functools

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .circuit import _here, _ptr

_REAL = {torch.float32: B.VQC_F32, torch.bfloat16: B.VQC_BF16, torch.float16: B.VQC_F16}


def _code(t, name):
    code = _REAL.get(t.dtype)
    if code is None or not t.is_cuda:
        raise ValueError("%s must be a CUDA float32, bfloat16 or float16 tensor (got %s %s)"
                         % (name, t.device, t.dtype))
    return code


def _out_code(dtype, out_dtype):
    if out_dtype not in _REAL or (out_dtype is not dtype and torch.float32 not in (dtype, out_dtype)):
        raise ValueError("the output of %s operands must be %s, float32 or, from float32, a 16-bit type (got %s)"
                         % (dtype, dtype, out_dtype))
    return _REAL[out_dtype]


def _act(activation):
    code = B.ACTIVATIONS.get(activation)
    if code is None:
        raise ValueError("activation must be one of %s (got %r)" % (sorted(B.ACTIVATIONS), activation))
    return code


def _rows(t, cols, name, dtype=None, rows=None):
    """(t as [rows, cols] with adjacent row elements, its row stride)."""
    if t.dim() == 0 or t.shape[-1] != cols or (dtype is not None and t.dtype is not dtype) or not t.is_cuda:
        raise ValueError("%s must be a CUDA %s tensor of shape [..., %d] (got %s %s %s)"
                         % (name, dtype or "", cols, t.device, t.dtype, tuple(t.shape)))
    if t.dim() != 2:
        t = t.reshape(-1, cols)
    if rows is not None and t.shape[0] != rows:
        raise ValueError("%s must have %d rows (got %d)" % (name, rows, t.shape[0]))
    ld, one = t.stride()
    if (one != 1 and cols > 1) or (ld < cols and t.shape[0] > 1):
        t, ld = t.contiguous(), cols
    return t, (ld if ld > cols else cols)


def _vector(t, n, dtype, name):
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.shape[0] != n or not t.is_cuda:
        raise ValueError("%s must be a CUDA %s tensor of shape (%d,) (got %s %s %s)"
                         % (name, dtype, n, t.device, t.dtype, tuple(t.shape)))
    return t if t.is_contiguous() else t.contiguous()


def _weight(t, cols, dtype, name):
    if t.dim() != 2 or t.shape[0] < 1:
        raise ValueError("%s must have two axes (got %s)" % (name, tuple(t.shape)))
    return _rows(t, cols, name, dtype)


def _sized(query):
    """A workspace query whose answers (functions of sizes, types and alignment) are kept."""
    @functools.lru_cache(maxsize=4096)
    def size(*args):
        nbytes = query(*args)
        if nbytes == 2 ** 64 - 1:
            raise ValueError("sizes out of range: %s" % (args,))
        return nbytes
    return size


_norm_bytes = _sized(B.vqc_layer_norm_workspace_bytes)
_linear_bytes = _sized(B.vqc_linear_workspace_bytes)
_gated_bytes = _sized(B.vqc_gated_workspace_bytes)


def _workspace(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None


def _aligned(*tensors):
    for t in tensors:
        if t.data_ptr() & 15:
            return 0
    return 1


# ------------------------------------------------------------------ layer norm

def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, save=True):
    """y, or (y, saved) where ``save``: saved holds the rows' mean and 1 / sqrt(var + eps)."""
    code, cols = _code(x, "x"), x.shape[-1] if x.dim() else 0
    x2, ld = _rows(x, cols, "x")
    weight, bias = _vector(weight, cols, x.dtype, "weight"), _vector(bias, cols, x.dtype, "bias")
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    stats = torch.empty(x2.shape[0], 2, dtype=torch.float32, device=x.device) if save else None
    B.vqc_layer_norm_forward(code, x2.shape[0], cols, x2.data_ptr(), ld, _ptr(weight), _ptr(bias), eps,
                             y.data_ptr(), _ptr(stats), _here()[1])
    return (y, stats) if save else y


def layer_norm_backward(grad_y, x, weight, saved, need_x=True, need_weight=True, need_bias=True):
    """(grad_x, grad_weight, grad_bias), None for those not needed."""
    code, cols = _code(x, "x"), x.shape[-1] if x.dim() else 0
    x2, ld = _rows(x, cols, "x")
    rows = x2.shape[0]
    gy, ld_gy = _rows(grad_y, cols, "grad_y", x.dtype, rows)
    weight = _vector(weight, cols, x.dtype, "weight")
    if saved.shape != (rows, 2) or saved.dtype is not torch.float32 or not saved.is_contiguous():
        raise ValueError("saved must be what layer_norm_forward returned for these rows")
    gx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
    gw = torch.empty(cols, dtype=x.dtype, device=x.device) if need_weight else None
    gb = torch.empty(cols, dtype=x.dtype, device=x.device) if need_bias else None
    ws, nbytes = None, 0
    if need_weight or need_bias:
        nbytes = _norm_bytes(rows, cols)
        ws = _workspace(nbytes)
    B.vqc_layer_norm_backward(code, rows, cols, gy.data_ptr(), ld_gy, x2.data_ptr(), ld, _ptr(weight),
                              saved.data_ptr(), _ptr(gx), _ptr(gw), _ptr(gb), _ptr(ws), nbytes,
                              _here()[1])
    return gx, gw, gb


class LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, stats = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, stats)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, weight, stats = ctx.saved_tensors
        need = ctx.needs_input_grad
        gx, gw, gb = layer_norm_backward(gy, x, weight, stats, need[0], need[1], need[2])
        return gx, gw, gb, None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last axis, differentiable in x, weight and bias."""
    return LayerNormFunction.apply(x, weight, bias, eps)


# ------------------------------------------------------------------ linear

def linear_forward(x, weight, bias=None, activation="none", residual=None, out_dtype=None, save=True):
    """y = act(x weight^T + bias) + residual, or (y, saved) where ``save``:
    saved holds the float32 pre-activations (None where there is no activation)."""
    code, act, cols = _code(x, "x"), _act(activation), x.shape[-1] if x.dim() else 0
    x2, ld = _rows(x, cols, "x")
    w, ld_w = _weight(weight, cols, x.dtype, "weight")
    rows, out = x2.shape[0], w.shape[0]
    bias = _vector(bias, out, x.dtype, "bias")
    y_type = x.dtype if out_dtype is None else out_dtype
    res, ld_res = (None, 0) if residual is None else _rows(residual, out, "residual", y_type, rows)
    y_code = _out_code(x.dtype, y_type)
    nbytes = _linear_bytes(0, code, y_code, rows, cols, out, ld, ld_w, 0, act, _aligned(x2, w))
    ws = _workspace(nbytes)
    y = torch.empty(x.shape[:-1] + (out,), dtype=y_type, device=x.device)
    z = torch.empty(rows, out, dtype=torch.float32, device=x.device) if save and act else None
    B.vqc_linear_forward(code, y_code, rows, cols, out, x2.data_ptr(), ld, w.data_ptr(), ld_w, _ptr(bias), act,
                         _ptr(res), ld_res, y.data_ptr(), _ptr(z), _ptr(ws), nbytes, _here()[1])
    return (y, z) if save else y


def linear_backward(grad_y, x, weight, saved, activation="none", need_x=True, need_weight=True, need_bias=True):
    """(grad_x, grad_weight, grad_bias), None for those not needed.  The
    residual's gradient is grad_y."""
    code, act, cols = _code(x, "x"), _act(activation), x.shape[-1] if x.dim() else 0
    x2, ld = _rows(x, cols, "x")
    w, ld_w = _weight(weight, cols, x.dtype, "weight")
    rows, out = x2.shape[0], w.shape[0]
    y_code = _out_code(x.dtype, grad_y.dtype)
    gy, ld_gy = _rows(grad_y, out, "grad_y", None, rows)
    if act and (saved is None or saved.shape != (rows, out) or saved.dtype is not torch.float32
                or not saved.is_contiguous()):
        raise ValueError("saved must be what linear_forward returned for these rows")
    gx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
    gw = torch.empty(out, cols, dtype=x.dtype, device=x.device) if need_weight else None
    gb = torch.empty(out, dtype=x.dtype, device=x.device) if need_bias else None
    nbytes = _linear_bytes(1, code, y_code, rows, cols, out, ld, ld_w, ld_gy, act, _aligned(x2, w, gy))
    ws = _workspace(nbytes)
    B.vqc_linear_backward(code, y_code, rows, cols, out, gy.data_ptr(), ld_gy, x2.data_ptr(), ld, w.data_ptr(),
                          ld_w, _ptr(saved), act, _ptr(gx), _ptr(gw), _ptr(gb), _ptr(ws), nbytes, _here()[1])
    return gx, gw, gb


class LinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, activation, residual, out_dtype):
        y, z = linear_forward(x, weight, bias, activation, residual, out_dtype)
        ctx.activation = activation
        ctx.save_for_backward(x, weight, z)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, gy):
        x, weight, z = ctx.saved_tensors
        need = ctx.needs_input_grad
        gx = gw = gb = None
        if need[0] or need[1] or need[2]:
            gx, gw, gb = linear_backward(gy, x, weight, z, ctx.activation, need[0], need[1], need[2])
        return gx, gw, gb, None, (gy if need[4] else None), None


def linear(x, weight, bias=None, activation="none", residual=None, out_dtype=None):
    """act(x weight^T + bias) + residual, differentiable in all four tensors.
    ``activation``: "none", "relu", "gelu", "silu", "tanh" or "sigmoid";
    ``out_dtype`` (and the residual's type) may be float32 for 16-bit x, or a
    16-bit type for float32 x."""
    return LinearFunction.apply(x, weight, bias, activation, residual, out_dtype)


# ------------------------------------------------------------------ gated

def _pair(weight_gate, weight_up, cols, dtype):
    if weight_gate.shape != weight_up.shape:
        raise ValueError("weight_gate and weight_up must have one shape (got %s and %s)"
                         % (tuple(weight_gate.shape), tuple(weight_up.shape)))
    wg, ld_g = _weight(weight_gate, cols, dtype, "weight_gate")
    wu, ld_u = _weight(weight_up, cols, dtype, "weight_up")
    if ld_g != ld_u:
        wg, wu, ld_g = wg.contiguous(), wu.contiguous(), cols
    return wg, wu, ld_g


def gated_forward(x, weight_gate, weight_up, bias_gate=None, bias_up=None, activation="silu", save=True):
    """h = act(g) * u, or (h, saved) where ``save``: saved holds g and u in float32."""
    code, act, cols = _code(x, "x"), _act(activation), x.shape[-1] if x.dim() else 0
    x2, ld = _rows(x, cols, "x")
    wg, wu, ld_w = _pair(weight_gate, weight_up, cols, x.dtype)
    rows, out = x2.shape[0], wg.shape[0]
    bg, bu = _vector(bias_gate, out, x.dtype, "bias_gate"), _vector(bias_up, out, x.dtype, "bias_up")
    nbytes = _gated_bytes(0, code, rows, cols, out, ld, ld_w, _aligned(x2, wg, wu))
    ws = _workspace(nbytes)
    h = torch.empty(x.shape[:-1] + (out,), dtype=x.dtype, device=x.device)
    z = torch.empty(2, rows, out, dtype=torch.float32, device=x.device) if save else None
    B.vqc_gated_forward(code, rows, cols, out, x2.data_ptr(), ld, wg.data_ptr(), wu.data_ptr(), ld_w, _ptr(bg),
                        _ptr(bu), act, h.data_ptr(), _ptr(z), _ptr(ws), nbytes, _here()[1])
    return (h, z) if save else h


def gated_backward(grad_h, x, weight_gate, weight_up, saved, activation="silu", need_x=True, need_weight=True,
                   need_bias=True):
    """(grad_x, grad_weight_gate, grad_weight_up, grad_bias_gate, grad_bias_up),
    None for those not needed."""
    code, act, cols = _code(x, "x"), _act(activation), x.shape[-1] if x.dim() else 0
    x2, ld = _rows(x, cols, "x")
    wg, wu, ld_w = _pair(weight_gate, weight_up, cols, x.dtype)
    rows, out = x2.shape[0], wg.shape[0]
    gh, ld_gh = _rows(grad_h, out, "grad_h", x.dtype, rows)
    if saved.shape != (2, rows, out) or saved.dtype is not torch.float32 or not saved.is_contiguous():
        raise ValueError("saved must be what gated_forward returned for these rows")
    gx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if need_x else None
    gw = [torch.empty(out, cols, dtype=x.dtype, device=x.device) if need_weight else None for _ in range(2)]
    gb = [torch.empty(out, dtype=x.dtype, device=x.device) if need_bias else None for _ in range(2)]
    nbytes = _gated_bytes(1, code, rows, cols, out, ld, ld_w, _aligned(x2, wg, wu))
    ws = _workspace(nbytes)
    B.vqc_gated_backward(code, rows, cols, out, gh.data_ptr(), ld_gh, x2.data_ptr(), ld, wg.data_ptr(),
                         wu.data_ptr(), ld_w, saved.data_ptr(), act, _ptr(gx), _ptr(gw[0]), _ptr(gw[1]),
                         _ptr(gb[0]), _ptr(gb[1]), _ptr(ws), nbytes, _here()[1])
    return gx, gw[0], gw[1], gb[0], gb[1]


class GatedFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight_gate, weight_up, bias_gate, bias_up, activation):
        h, z = gated_forward(x, weight_gate, weight_up, bias_gate, bias_up, activation)
        ctx.activation = activation
        ctx.save_for_backward(x, weight_gate, weight_up, z)
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, gh):
        x, wg, wu, z = ctx.saved_tensors
        need = ctx.needs_input_grad
        got = gated_backward(gh, x, wg, wu, z, ctx.activation, need[0], need[1] or need[2], need[3] or need[4])
        return tuple(g if n else None for g, n in zip(got, need)) + (None,)


def gated(x, weight_gate, weight_up, bias_gate=None, bias_up=None, activation="silu"):
    """act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up), both
    projections, the activation and the product in one kernel; differentiable
    in all five tensors."""
    return GatedFunction.apply(x, weight_gate, weight_up, bias_gate, bias_up, activation)
