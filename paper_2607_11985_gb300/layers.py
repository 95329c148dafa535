"""Classical operators of a hybrid model, for torch CUDA tensors.

What stands around a ``Circuit`` inside a network, in the library's kernels:

  layer_norm   y = (x - mean) / sqrt(var + eps) * weight + bias over the last axis
  linear       y = act(x weight^T + bias) + residual: features to a circuit's
               angles, expectations back to features, ordinary projections
  gated        h = act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up)

Each has three forms: ``linear_forward`` and ``linear_backward`` are the two
calls of a training step (or inference with ``save=False``), ``linear`` the
same under autograd (once; forward-mode derivatives are refused).  x may have
any leading axes; rows may be strided (other layouts are copied).  Types:
float32, bfloat16 and float16, sums and statistics in float; see include/vqc.h
for the formulas and roundings.  Tensors are on the current device, work goes to
its current stream.  Torch supplies device memory and the stream only.
Arguments that do not fit raise ValueError, statuses of the library
``binding.VQCError``.  A product whose waits ran out (VQC_WAIT_NS, 4 s) leaves its
output incomplete: later calls raise until ``binding.vqc_sync_check`` has been told.

A call on a few rows costs its host path, so the checks, the allocations and the
calls of the C entry points are native (csrc/layers_torch.cpp, ``_layers.so``).
"""
from __future__ import annotations

import torch

from . import binding as B

B.lib()                      # fails loudly where the library is not built

from . import _layers as _native   # noqa: E402

_REAL = {torch.float32: B.VQC_F32, torch.bfloat16: B.VQC_BF16, torch.float16: B.VQC_F16, None: -1}
_ACT = B.ACTIVATIONS


def _act(activation):
    code = _ACT.get(activation)
    if code is None:
        raise ValueError("activation must be one of %s (got %r)" % (sorted(_ACT), activation))
    return code


def _type(dtype):
    code = _REAL.get(dtype)
    if code is None:
        raise ValueError("out_dtype must be float32, bfloat16 or float16 (got %s)" % (dtype,))
    return code


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, save=True):
    """y, or (y, saved) where ``save``: saved holds the rows' mean and 1 / sqrt(var + eps)."""
    return _native.norm_forward(x, weight, bias, eps, save)


def layer_norm_backward(grad_y, x, weight, saved, need_x=True, need_weight=True, need_bias=True):
    """(grad_x, grad_weight, grad_bias), None for those not needed."""
    return _native.norm_backward(grad_y, x, weight, saved, need_x, need_weight, need_bias)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last axis, differentiable in x, weight and bias."""
    return _native.norm(x, weight, bias, eps)


def linear_forward(x, weight, bias=None, activation="none", residual=None, out_dtype=None, save=True):
    """y = act(x weight^T + bias) + residual, or (y, saved) where ``save``:
    saved holds the float32 pre-activations (None where there is no activation)."""
    return _native.linear_forward(x, weight, bias, _act(activation), residual, _type(out_dtype), save)


def linear_backward(grad_y, x, weight, saved, activation="none", need_x=True, need_weight=True, need_bias=True):
    """(grad_x, grad_weight, grad_bias), None for those not needed.  The
    residual's gradient is grad_y."""
    return _native.linear_backward(grad_y, x, weight, saved, _act(activation), need_x, need_weight, need_bias)


def linear(x, weight, bias=None, activation="none", residual=None, out_dtype=None):
    """act(x weight^T + bias) + residual, differentiable in all four tensors.
    The residual has as many rows as x, in any leading axes.
    ``activation``: "none", "relu", "gelu", "silu", "tanh" or "sigmoid";
    ``out_dtype`` (and the residual's type) may be float32 for 16-bit x, or a
    16-bit type for float32 x."""
    return _native.linear(x, weight, bias, _act(activation), residual, _type(out_dtype))


def gated_forward(x, weight_gate, weight_up, bias_gate=None, bias_up=None, activation="silu", save=True):
    """h = act(g) * u, or (h, saved) where ``save``: saved holds g and u in float32."""
    return _native.gated_forward(x, weight_gate, weight_up, bias_gate, bias_up, _act(activation), save)


def gated_backward(grad_h, x, weight_gate, weight_up, saved, activation="silu", need_x=True, need_weight=True,
                   need_bias=True):
    """(grad_x, grad_weight_gate, grad_weight_up, grad_bias_gate, grad_bias_up),
    None for those not needed."""
    return _native.gated_backward(grad_h, x, weight_gate, weight_up, saved, _act(activation), need_x, need_weight,
                                  need_bias)


def gated(x, weight_gate, weight_up, bias_gate=None, bias_up=None, activation="silu"):
    """act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up), both
    projections, the activation and the product in one kernel; differentiable
    in all five tensors."""
    return _native.gated(x, weight_gate, weight_up, bias_gate, bias_up, _act(activation))
