"""Classical operators of a hybrid model, for torch CUDA tensors.

What stands around a ``Circuit`` inside a network, in the library's kernels:

  layer_norm   y = (x - mean) / sqrt(var + eps) * weight + bias over the last axis
  linear       y = act(x weight^T + bias) + residual: features to a circuit's
               angles, expectations back to features, ordinary projections
  gated        h = act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up)

Each has three forms: ``linear_forward`` and ``linear_backward`` are the two
calls of a training step (or inference with ``save=False``), ``linear`` the
same under autograd.  x may have any leading axes; rows may be strided (other
layouts are copied).  Types: float32, bfloat16 and float16, sums and
statistics in float; see include/vqc.h for the formulas and roundings.  Tensors
are on the current device, work goes to its current stream.  Torch supplies
device memory and the stream only.

A call on a few rows costs its host path, so that is kept short: checks are one
test each where they pass, and the C entry points are called directly.
"""
from __future__ import annotations

import functools

import torch
from torch.autograd.function import once_differentiable

from . import binding as B
from .circuit import _raw_stream

_REAL = {torch.float32: B.VQC_F32, torch.bfloat16: B.VQC_BF16, torch.float16: B.VQC_F16}
_ACT = B.ACTIVATIONS
_F32 = torch.float32
_empty = torch.empty
_device = torch.cuda.current_device


def _matrix(t, name):
    """(type code, t as [rows, cols] with adjacent row elements, rows, cols, row stride)."""
    code = _REAL.get(t.dtype)
    if code is None or t.get_device() != _device() or t.dim() == 0:
        raise ValueError("%s must be a CUDA float32, bfloat16 or float16 tensor on the current device (got %s %s %s)"
                         % (name, t.device, t.dtype, tuple(t.shape)))
    if t.dim() != 2:
        t = t.reshape(-1, t.shape[-1])
    rows, cols = t.shape
    if t.is_contiguous():
        return code, t, rows, cols, cols
    ld, one = t.stride()
    if (one != 1 and cols > 1) or (ld < cols and rows > 1):
        return code, t.contiguous(), rows, cols, cols
    return code, t, rows, cols, max(ld, cols)


def _like(t, rows, cols, code, name):
    """(t as a matrix, its row stride), t of the given sizes and type (None: any type)."""
    got, t, r, c, ld = _matrix(t, name)
    if (r != rows and rows is not None) or c != cols or (got != code and code is not None):
        raise ValueError("%s must have %s rows of %d elements and the operands' type (got %s %s)"
                         % (name, rows, cols, tuple(t.shape), t.dtype))
    return t, ld


def _weight(t, cols, code, name):
    if t.dim() != 2 or t.shape[0] < 1:
        raise ValueError("%s must have two axes (got %s)" % (name, tuple(t.shape)))
    return _like(t, None, cols, code, name)


def _vector(t, n, dtype, name):
    """(t, its address), or Nones."""
    if t is None:
        return None, None
    if t.dtype is not dtype or t.shape != (n,) or not t.is_cuda:
        raise ValueError("%s must be a CUDA %s tensor of shape (%d,) (got %s %s %s)"
                         % (name, dtype, n, t.device, t.dtype, tuple(t.shape)))
    if not t.is_contiguous():
        t = t.contiguous()
    return t, t.data_ptr()


def _saved(t, shape):
    if t is None or t.shape != shape or t.dtype is not _F32 or not t.is_contiguous():
        raise ValueError("saved must be what the forward returned for these rows")
    return t.data_ptr()


def _out_code(dtype, out_dtype):
    code = _REAL.get(out_dtype)
    if code is None or (out_dtype is not dtype and _F32 not in (dtype, out_dtype)):
        raise ValueError("the output of %s operands must be %s, float32 or, from float32, a 16-bit type (got %s)"
                         % (dtype, dtype, out_dtype))
    return code


def _act(activation):
    code = _ACT.get(activation)
    if code is None:
        raise ValueError("activation must be one of %s (got %r)" % (sorted(_ACT), activation))
    return code


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
    """(a workspace, its address): fresh for every call, so that calls of several
    threads and streams never share one."""
    if nbytes == 0:
        return None, None
    ws = _empty(nbytes, dtype=torch.uint8, device="cuda")
    return ws, ws.data_ptr()


def _new(need, shape, like):
    """(an output tensor of like's type, its address), or Nones."""
    if not need:
        return None, None
    t = like.new_empty(shape)
    return t, t.data_ptr()


def _stream():
    return _raw_stream(_device())


# ------------------------------------------------------------------ layer norm

def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, save=True):
    """y, or (y, saved) where ``save``: saved holds the rows' mean and 1 / sqrt(var + eps)."""
    code, x2, rows, cols, ld = _matrix(x, "x")
    weight, pw = _vector(weight, cols, x.dtype, "weight")
    bias, pb = _vector(bias, cols, x.dtype, "bias")
    y, py = _new(True, x.shape, x)
    stats = _empty(rows, 2, dtype=_F32, device=x.device) if save else None
    st = B.lib().vqc_layer_norm_forward(code, rows, cols, x2.data_ptr(), ld, pw, pb, eps, py,
                                        stats.data_ptr() if save else None, _stream())
    if st:
        B._check(st)
    return (y, stats) if save else y


def layer_norm_backward(grad_y, x, weight, saved, need_x=True, need_weight=True, need_bias=True):
    """(grad_x, grad_weight, grad_bias), None for those not needed."""
    code, x2, rows, cols, ld = _matrix(x, "x")
    gy, ld_gy = _like(grad_y, rows, cols, code, "grad_y")
    weight, pw = _vector(weight, cols, x.dtype, "weight")
    stats = _saved(saved, (rows, 2))
    gx, px = _new(need_x, x.shape, x)
    gw, pgw = _new(need_weight, cols, x)
    gb, pgb = _new(need_bias, cols, x)
    nbytes = _norm_bytes(rows, cols) if need_weight or need_bias else 0
    ws, pws = _workspace(nbytes)
    st = B.lib().vqc_layer_norm_backward(code, rows, cols, gy.data_ptr(), ld_gy, x2.data_ptr(), ld, pw, stats, px, pgw,
                                         pgb, pws, nbytes, _stream())
    if st:
        B._check(st)
    return gx, gw, gb


def _norm_gradients(ctx, gy):
    x, weight, stats = ctx.saved_tensors
    need = ctx.needs_input_grad
    gx, gw, gb = layer_norm_backward(gy, x, weight, stats, need[0], need[1], need[2])
    return gx, gw, gb, None


class LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, stats = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, stats)
        return y

    backward = staticmethod(once_differentiable(_norm_gradients))


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last axis, differentiable in x, weight and bias."""
    return LayerNormFunction.apply(x, weight, bias, eps)


# ------------------------------------------------------------------ linear

def linear_forward(x, weight, bias=None, activation="none", residual=None, out_dtype=None, save=True):
    """y = act(x weight^T + bias) + residual, or (y, saved) where ``save``:
    saved holds the float32 pre-activations (None where there is no activation)."""
    act = _act(activation)
    code, x2, rows, cols, ld = _matrix(x, "x")
    w, ld_w = _weight(weight, cols, code, "weight")
    out = w.shape[0]
    bias, pb = _vector(bias, out, x.dtype, "bias")
    y_type, y_code = (x.dtype, code) if out_dtype is None else (out_dtype, _out_code(x.dtype, out_dtype))
    res = pr = None
    ld_res = 0
    if residual is not None:
        res, ld_res = _like(residual, rows, out, y_code, "residual")
        pr = res.data_ptr()
    px, pw = x2.data_ptr(), w.data_ptr()
    nbytes = _linear_bytes(0, code, y_code, rows, cols, out, ld, ld_w, 0, act, 0 if (px | pw) & 15 else 1)
    ws, pws = _workspace(nbytes)
    y = _empty(x.shape[:-1] + (out,), dtype=y_type, device=x.device)
    z = _empty(rows, out, dtype=_F32, device=x.device) if save and act else None
    st = B.lib().vqc_linear_forward(code, y_code, rows, cols, out, px, ld, pw, ld_w, pb, act, pr, ld_res, y.data_ptr(),
                                    None if z is None else z.data_ptr(), pws, nbytes, _stream())
    if st:
        B._check(st)
    return (y, z) if save else y


def linear_backward(grad_y, x, weight, saved, activation="none", need_x=True, need_weight=True, need_bias=True):
    """(grad_x, grad_weight, grad_bias), None for those not needed.  The
    residual's gradient is grad_y."""
    act = _act(activation)
    code, x2, rows, cols, ld = _matrix(x, "x")
    w, ld_w = _weight(weight, cols, code, "weight")
    out = w.shape[0]
    y_code = _out_code(x.dtype, grad_y.dtype)
    gy, ld_gy = _like(grad_y, rows, out, y_code, "grad_y")
    pz = _saved(saved, (rows, out)) if act else None
    gx, pgx = _new(need_x, x.shape, x)
    gw, pgw = _new(need_weight, (out, cols), x)
    gb, pgb = _new(need_bias, out, x)
    px, pw, pg = x2.data_ptr(), w.data_ptr(), gy.data_ptr()
    nbytes = _linear_bytes(1, code, y_code, rows, cols, out, ld, ld_w, ld_gy, act, 0 if (px | pw | pg) & 15 else 1)
    ws, pws = _workspace(nbytes)
    st = B.lib().vqc_linear_backward(code, y_code, rows, cols, out, pg, ld_gy, px, ld, pw, ld_w, pz, act, pgx, pgw, pgb,
                                     pws, nbytes, _stream())
    if st:
        B._check(st)
    return gx, gw, gb


def _linear_gradients(ctx, gy):
    x, weight, z = ctx.saved_tensors
    need = ctx.needs_input_grad
    gx = gw = gb = None
    if need[0] or need[1] or need[2]:
        gx, gw, gb = linear_backward(gy, x, weight, z, ctx.activation, need[0], need[1], need[2])
    return gx, gw, gb, None, (gy if need[4] else None), None


class LinearFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, activation, residual, out_dtype):
        y, z = linear_forward(x, weight, bias, activation, residual, out_dtype)
        ctx.activation = activation
        ctx.save_for_backward(x, weight, z)
        return y

    backward = staticmethod(once_differentiable(_linear_gradients))


def linear(x, weight, bias=None, activation="none", residual=None, out_dtype=None):
    """act(x weight^T + bias) + residual, differentiable in all four tensors.
    ``activation``: "none", "relu", "gelu", "silu", "tanh" or "sigmoid";
    ``out_dtype`` (and the residual's type) may be float32 for 16-bit x, or a
    16-bit type for float32 x."""
    return LinearFunction.apply(x, weight, bias, activation, residual, out_dtype)


# ------------------------------------------------------------------ gated

def _pair(weight_gate, weight_up, cols, code):
    if weight_gate.shape != weight_up.shape:
        raise ValueError("weight_gate and weight_up must have one shape (got %s and %s)"
                         % (tuple(weight_gate.shape), tuple(weight_up.shape)))
    wg, ld_g = _weight(weight_gate, cols, code, "weight_gate")
    wu, ld_u = _weight(weight_up, cols, code, "weight_up")
    if ld_g != ld_u:
        wg, wu, ld_g = wg.contiguous(), wu.contiguous(), cols
    return wg, wu, ld_g


def gated_forward(x, weight_gate, weight_up, bias_gate=None, bias_up=None, activation="silu", save=True):
    """h = act(g) * u, or (h, saved) where ``save``: saved holds g and u in float32."""
    act = _act(activation)
    code, x2, rows, cols, ld = _matrix(x, "x")
    wg, wu, ld_w = _pair(weight_gate, weight_up, cols, code)
    out = wg.shape[0]
    bias_gate, pbg = _vector(bias_gate, out, x.dtype, "bias_gate")
    bias_up, pbu = _vector(bias_up, out, x.dtype, "bias_up")
    px, pwg, pwu = x2.data_ptr(), wg.data_ptr(), wu.data_ptr()
    nbytes = _gated_bytes(0, code, rows, cols, out, ld, ld_w, 0 if (px | pwg | pwu) & 15 else 1)
    ws, pws = _workspace(nbytes)
    h, ph = _new(True, x.shape[:-1] + (out,), x)
    z = _empty(2, rows, out, dtype=_F32, device=x.device) if save else None
    st = B.lib().vqc_gated_forward(code, rows, cols, out, px, ld, pwg, pwu, ld_w, pbg, pbu, act, ph,
                                   None if z is None else z.data_ptr(), pws, nbytes, _stream())
    if st:
        B._check(st)
    return (h, z) if save else h


def gated_backward(grad_h, x, weight_gate, weight_up, saved, activation="silu", need_x=True, need_weight=True,
                   need_bias=True):
    """(grad_x, grad_weight_gate, grad_weight_up, grad_bias_gate, grad_bias_up),
    None for those not needed."""
    act = _act(activation)
    code, x2, rows, cols, ld = _matrix(x, "x")
    wg, wu, ld_w = _pair(weight_gate, weight_up, cols, code)
    out = wg.shape[0]
    gh, ld_gh = _like(grad_h, rows, out, code, "grad_h")
    pz = _saved(saved, (2, rows, out))
    gx, pgx = _new(need_x, x.shape, x)
    gwg, pgwg = _new(need_weight, (out, cols), x)
    gwu, pgwu = _new(need_weight, (out, cols), x)
    gbg, pgbg = _new(need_bias, out, x)
    gbu, pgbu = _new(need_bias, out, x)
    px, pwg, pwu, pg = x2.data_ptr(), wg.data_ptr(), wu.data_ptr(), gh.data_ptr()
    nbytes = _gated_bytes(1, code, rows, cols, out, ld, ld_w, 0 if (px | pwg | pwu | pg) & 15 else 1)
    ws, pws = _workspace(nbytes)
    st = B.lib().vqc_gated_backward(code, rows, cols, out, pg, ld_gh, px, ld, pwg, pwu, ld_w, pz, act, pgx, pgwg, pgwu,
                                    pgbg, pgbu, pws, nbytes, _stream())
    if st:
        B._check(st)
    return gx, gwg, gwu, gbg, gbu


def _gated_gradients(ctx, gh):
    x, wg, wu, z = ctx.saved_tensors
    need = ctx.needs_input_grad
    got = gated_backward(gh, x, wg, wu, z, ctx.activation, need[0], need[1] or need[2], need[3] or need[4])
    return tuple(g if n else None for g, n in zip(got, need)) + (None,)


class GatedFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight_gate, weight_up, bias_gate, bias_up, activation):
        h, z = gated_forward(x, weight_gate, weight_up, bias_gate, bias_up, activation)
        ctx.activation = activation
        ctx.save_for_backward(x, weight_gate, weight_up, z)
        return h

    backward = staticmethod(once_differentiable(_gated_gradients))


def gated(x, weight_gate, weight_up, bias_gate=None, bias_up=None, activation="silu"):
    """act(x weight_gate^T + bias_gate) * (x weight_up^T + bias_up), both
    projections, the activation and the product in one kernel; differentiable
    in all five tensors."""
    return GatedFunction.apply(x, weight_gate, weight_up, bias_gate, bias_up, activation)
