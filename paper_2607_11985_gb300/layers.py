"""Classical operators of a hybrid model, for torch CUDA tensors.

What stands around a ``Circuit`` inside a network, in the library's kernels:

  layer_norm   y = (x - mean) / sqrt(var + eps) * weight + bias over the last axis
  linear       y = act(x weight^T + bias) + residual: features to a circuit's
               angles, expectations back to features, ordinary projections
  gated        h = act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up)
  dropout      y = residual + x / (1 - p) where an element is kept, from a counter-based
               generator: no mask is stored
  norm_rotary  queries and keys [batch, tokens, heads, dim]: a norm of each head, and
               pairs of its elements turned by position * frequency
  attention    causal attention through a window and over the first tokens (sinks);
               query heads share key heads

Each has three forms: ``linear_forward`` and ``linear_backward`` are the two
calls of a training step (or inference with ``save=False``), ``linear`` the
same under autograd (once; forward-mode derivatives are refused).  ``norm_rotary_step`` and
``attention_step`` are the forms for serving: the last tokens of sequences, over a cache of their keys
and values.  x may have any leading axes; rows may be strided (other layouts are copied).  Types:
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


def dropout_forward(x, p, seed, offset=0, residual=None):
    """residual + x / (1 - p) where an element is kept, residual (or 0) where it is not.
    Element e (in rows) is kept where word e % 4 of Philox 4x32-10 at counter (e / 4, offset) and key
    ``seed`` is at least p 2^32.  ``seed``: an integer (64 bits of it count), or a CUDA int64
    tensor (seed, offset) that is read when the kernel runs (``offset`` is added), so that a captured call
    draws anew in every replay.  Layers and steps that share a seed need offsets of their own."""
    return _native.dropout_forward(x, p, seed, offset, residual)


def dropout_backward(grad_y, p, seed, offset=0):
    """grad_x: the same elements are drawn again.  The residual's gradient is grad_y."""
    return _native.dropout_backward(grad_y, p, seed, offset)


def dropout(x, p, seed, offset=0, residual=None):
    """See ``dropout_forward``; differentiable in x and the residual.  (In training: evaluation
    is the residual's sum alone.)"""
    return _native.dropout(x, p, seed, offset, residual)


def rotary_frequencies(dim, base=10000.0, device="cuda"):
    """Radians per position of the dim / 2 pairs of a head whose first ``dim`` elements are turned:
    base^(-2 i / dim), in float64."""
    if dim < 2 or dim % 2:
        raise ValueError("dim must be even and positive (got %r)" % (dim,))
    return torch.tensor([base ** (-2.0 * i / dim) for i in range(dim // 2)], dtype=torch.float64, device=device)


def norm_rotary_forward(q, k, weight_q=None, weight_k=None, frequencies=None, positions=None, eps=1e-6):
    """(q', k') dense: x / sqrt(mean(x^2) + eps) * weight of each head, then its pairs (i, n + i) turned by
    position * frequencies[i], n = len(frequencies) <= dim / 2 (None: nothing is turned).  q [batch, tokens,
    heads, dim], k [batch, tokens, groups, dim] may be slices of a wider tensor; dim up to 256.
    positions: int32 [batch, tokens] or [tokens], by default 0, 1, .."""
    return _native.rotary_forward(q, k, weight_q, weight_k, frequencies, positions, eps)


def norm_rotary_backward(grad_q, grad_k, q, k, weight_q=None, weight_k=None, frequencies=None, positions=None, eps=1e-6,
                         need_x=True, need_weight=True):
    """Gradients of (q, k, weight_q, weight_k), None for those not needed.  Nothing is saved by the forward."""
    return _native.rotary_backward(grad_q, grad_k, q, k, weight_q, weight_k, frequencies, positions, eps, need_x, need_weight)


def norm_rotary(q, k, weight_q=None, weight_k=None, frequencies=None, positions=None, eps=1e-6):
    """See ``norm_rotary_forward``; differentiable in q, k and the weights (frequencies that need a gradient are refused)."""
    return _native.rotary(q, k, weight_q, weight_k, frequencies, positions, eps)


def norm_rotary_step(q, k, v, cache_k, cache_v, lengths, weight_q=None, weight_k=None, frequencies=None, eps=1e-6):
    """q' of new tokens, whose k' and v are written into the caches [batch, capacity, groups, dim] in place:
    token t of a sequence stands at position lengths - tokens + t (lengths: int32 [batch], with the
    new tokens); places outside of the cache are not written.  The caches must lie apart from
    each other (views of one tensor that holds both are fine where their places are others) and from q, k and v.  No
    gradients: tensors that need one are refused while autograd records."""
    return _native.rotary_step(q, k, v, cache_k, cache_v, lengths, weight_q, weight_k, frequencies, eps)


def attention_forward(q, k, v, window=None, sinks=0, scale=None, lengths=None, save=True):
    """o [batch, tokens, heads, dim], or (o, saved) where ``save``: query i sees key j where j <= i and
    (i - j < window or j < sinks), both below the sequence's length.  k, v [batch, tokens, groups, dim]: head
    h reads group h / (heads / groups); dim up to 256.  window None: every earlier position; scale None:
    1 / sqrt(dim); lengths: int32 [batch] of padded sequences (rows from there on are zero), None: all tokens.
    saved holds the float32 log of the sum of exponentials of each row."""
    return _native.attention_forward(q, k, v, window, sinks, scale, lengths, save)


def attention_backward(grad_o, q, k, v, o, saved, window=None, sinks=0, scale=None, lengths=None, need_q=True, need_kv=True):
    """(grad_q, grad_k, grad_v), None for those not needed."""
    return _native.attention_backward(grad_o, q, k, v, o, saved, window, sinks, scale, lengths, need_q, need_kv)


def attention(q, k, v, window=None, sinks=0, scale=None, lengths=None):
    """See ``attention_forward``; differentiable in q, k and v."""
    return _native.attention(q, k, v, window, sinks, scale, lengths)


def attention_step(q, cache_k, cache_v, lengths, window=None, sinks=0, scale=None):
    """o of the last tokens of sequences over caches [batch, capacity, groups, dim]: token t stands at
    position lengths - tokens + t (lengths: int32 [batch], the tokens in the cache) and sees what ``attention`` sees
    there.  No gradients: tensors that need one are refused while autograd records."""
    return _native.attention_step(q, cache_k, cache_v, window, sinks, scale, lengths)
