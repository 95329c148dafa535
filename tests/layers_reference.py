"""The classical operators in 64 bits, with bounds on what the kernels may be off.

Every function returns {name: (value, bound)}: the float64 result of the
definition on the given (already rounded) inputs, and an elementwise bound that
follows from the roundings that the kernels make: float sums of n terms
(n + 2 roundings of at most 2^-23 of the sum of magnitudes: the tensor cores may
cut where float32 rounds), functions of the math library (2^-20), one rounding of
dz to 16 bits before the products of the backward, one rounding of each result.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
SUM, LIB = 2.0 ** -23, 2.0 ** -20
SLOPE, BEND = 1.2, 1.0          # the largest |act'| and |act''| of the activations


def act(name, z):
    """(act(z), act'(z)) in float64."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if name == "tanh":
        return torch.tanh(z), 1.0 - torch.tanh(z) ** 2
    if name == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    p = torch.sigmoid(z)
    if name == "sigmoid":
        return p, p * (1.0 - p)
    return z * p, p * (1.0 + z * (1.0 - p))


def rounded(v, e, dtype):
    return v, e + U[dtype] * (v.abs() + e) + TINY[dtype]


def project(x, w, b):
    z = x @ w.t() + (0.0 if b is None else b)
    size = x.abs() @ w.abs().t() + (0.0 if b is None else b.abs())
    return z, (x.shape[1] + 2) * SUM * size


def act_bounds(name, z, ez):
    """act and act' with their bounds, z known to ez."""
    a, d = act(name, z)
    ea = SLOPE * ez + LIB * (a.abs() + ez)
    ed = BEND * ez + LIB * (1.0 + z.abs()) if name != "none" else torch.zeros_like(z)
    if name == "relu":
        ed = (z.abs() <= ez).double()
    return a, ea, d, ed


def product(a, ea, b, eb, count, dtype):
    """a @ b of operands known to ea, eb, float sums of `count` terms, one rounding."""
    v = a @ b
    e = ea @ b.abs() + a.abs() @ eb + ea @ eb + (count + 2) * SUM * (a.abs() @ b.abs())
    return rounded(v, e, dtype)


def column_sum(d, ed, dtype):
    return rounded(d.sum(0), ed.sum(0) + (d.shape[0] + 2) * SUM * d.abs().sum(0), dtype)


def linear(x, w, b, name, res, gy, dtype, out_dtype):
    z, ez = project(x, w, b)
    a, ea, d, ed = act_bounds(name, z, ez)
    y = a if res is None else a + res
    out = {"y": rounded(y, ea + SUM * y.abs(), out_dtype), "z": (z, ez)}
    if gy is not None:
        dz, edz = gy * d, gy.abs() * ed + SUM * (gy * d).abs()
        exact = name == "none" and dtype == out_dtype
        dzr, edzr = (dz, edz) if dtype == torch.float32 or exact else rounded(dz, edz, dtype)
        zero = torch.zeros_like
        out["gx"] = product(dzr, edzr, w, zero(w), w.shape[0], dtype)
        out["gw"] = product(dzr.t(), edzr.t(), x, zero(x), x.shape[0], dtype)
        out["gb"] = column_sum(dz, edz, dtype)
    return out


def gated(x, wg, wu, bg, bu, name, gh, dtype):
    g, eg = project(x, wg, bg)
    u, eu = project(x, wu, bu)
    a, ea, d, ed = act_bounds(name, g, eg)
    h = a * u
    out = {"y": rounded(h, ea * u.abs() + a.abs() * eu + ea * eu + SUM * h.abs(), dtype)}
    if gh is not None:
        dg, du = gh * u * d, gh * a
        edg = gh.abs() * (eu * d.abs() + (u.abs() + eu) * ed) + 2 * SUM * dg.abs()
        edu = gh.abs() * ea + SUM * du.abs()
        dgr, edgr = (dg, edg) if dtype == torch.float32 else rounded(dg, edg, dtype)
        dur, edur = (du, edu) if dtype == torch.float32 else rounded(du, edu, dtype)
        both, eboth, wide = torch.cat([dgr, dur], 1), torch.cat([edgr, edur], 1), torch.cat([wg, wu], 0)
        out["gx"] = product(both, eboth, wide, torch.zeros_like(wide), wide.shape[0], dtype)
        out["gw"] = product(dgr.t(), edgr.t(), x, torch.zeros_like(x), x.shape[0], dtype)
        out["gup"] = product(dur.t(), edur.t(), x, torch.zeros_like(x), x.shape[0], dtype)
        out["gb"], out["gbup"] = column_sum(dg, edg, dtype), column_sum(du, edu, dtype)
    return out


def layer_norm(x, w, b, eps, gy, dtype):
    n, u = x.shape[1], 2.0 ** -24
    mean = x.mean(1, keepdim=True)
    r = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    em = (n + 2) * u * x.abs().mean(1, keepdim=True)
    er = 0.5 * (n + 6) * u + 0.5 * (r * em) ** 2 + 4 * u      # relative, of r
    h = (x - mean) * r
    eh = r * em + h.abs() * (er + 4 * u)
    wv = torch.ones(n, dtype=torch.float64) if w is None else w
    y = h * wv + (0.0 if b is None else b)
    out = {"y": rounded(y, eh * wv.abs() + 2 * u * (h * wv).abs() + 2 * u * y.abs(), dtype)}
    if gy is not None:
        g = gy * wv
        s, t = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
        es = (n + 4) * u * g.abs().mean(1, keepdim=True)
        et = (n + 4) * u * (g * h).abs().mean(1, keepdim=True) + (g.abs() * eh).mean(1, keepdim=True)
        inner = g - s - h * t
        e = r * (4 * u * (g.abs() + s.abs() + (h * t).abs()) + es + h.abs() * et + eh * t.abs() + eh * et)
        out["gx"] = rounded(r * inner, e + (r * inner).abs() * er, dtype)
        out["gw"] = column_sum(gy * h, gy.abs() * eh + u * (gy * h).abs(), dtype)
        out["gb"] = column_sum(gy, torch.zeros_like(gy), dtype)
    return out


def check(got, want, dtype, roundings, what):
    """Elementwise against the bound, and as a whole: the 2-norm of the error may be
    `roundings` roundings of the result's (plus 2e-6 of float work)."""
    value, bound = want
    d = (got.detach().double().cpu() - value).abs()
    assert got.shape == value.shape, (what, got.shape, value.shape)
    bad = ~(d <= bound)
    assert not bad.any(), "%s: %d of %d outside, worst %g at bound %g" % (
        what, int(bad.sum()), d.numel(), float((d / bound).nan_to_num(math.inf).max()), float(bound.max()))
    norm = float(value.norm())
    if d.numel() >= 4096 and norm > 0:
        rel = float(d.norm()) / norm
        assert rel <= roundings * U[dtype] + 2e-6, "%s: relative error %g" % (what, rel)
