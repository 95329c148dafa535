"""The operators of a sequence in 64 bits, with bounds on what the kernels may be off.

As layers_reference: {name: (value, bound)}, bounds from the roundings that the kernels make.  For
attention: scores are float sums of dim terms; a probability has the relative error of its score (twice: in it
and in its row's sum), of the library's exp2 (2^-20 with the arguments' roundings), and one rounding to 16 bits;
d = g . o is taken from the rounded o; ds is rounded to 16 bits once more.
"""
import math

import numpy as np
import torch

from tests.layers_reference import LIB, SUM, U, rounded

FLOAT = 2.0 ** -24


def philox(block, offset, seed):
    """Philox 4x32-10 (Salmon et al. 2011): four words for each 64-bit block."""
    m, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    block = np.asarray(block, dtype=np.uint64)
    c = [block & m, block >> half, np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    for r in range(10):
        k0 = np.uint64(((seed & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> half) ^ c[1] ^ k0, b & m, (a >> half) ^ c[3] ^ k1, a & m]
    return np.stack(c, -1)


def kept(shape, p, seed, offset):
    n = math.prod(shape)
    words = philox(np.arange((n + 3) // 4), offset % 2 ** 64, seed % 2 ** 64).reshape(-1)[:n]
    return torch.from_numpy((words >= np.uint64(min(round(p * 2 ** 32), 2 ** 32 - 1))).reshape(shape))


def dropout(x, res, gy, p, seed, offset, dtype):
    """x, res, gy in float64 on the CPU"""
    on = kept(x.shape, p, seed, offset)
    y = torch.where(on, x / (1 - p), 0.0)
    scaled = y.abs() * 2 * FLOAT          # of the factor, and of the product
    y = y + (0.0 if res is None else res)
    gx = torch.where(on, gy / (1 - p), 0.0)
    return {"y": rounded(y, scaled + FLOAT * y.abs(), dtype), "gx": rounded(gx, gx.abs() * 2 * FLOAT, dtype)}


# -------------------------------------------------------------- norms and rotation

def turn(a, b, c, s):
    return a * c - b * s, b * c + a * s


def norm_rotary(x, w, freq, pos, eps, g, dtype):
    """x, g [batch, tokens, heads, dim] in float64; pos [batch, tokens]; w [dim] or None"""
    n, dim = 0 if freq is None else freq.numel(), x.shape[-1]
    wv = torch.ones(dim, dtype=torch.float64) if w is None else w
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    m = x * r
    em = (0.5 * (dim + 6) + 4) * FLOAT * m.abs()               # r: half the sum's error, rsqrt
    h, eh = m * wv, em * wv.abs() + 2 * FLOAT * (m * wv).abs()
    if n:
        angle = (pos.double()[..., None] * freq)[:, :, None]
        c, s = torch.cos(angle), torch.sin(angle)
        ec = math.pi * FLOAT + 4 * FLOAT + angle.abs() * 2.0 ** -52      # float argument, sincospi, the frequency's rounding
    def turned(v, ev, back):
        if not n:
            return v, ev
        sign = -s if back else s
        a, b, ea, eb = v[..., :n], v[..., n:2 * n], ev[..., :n], ev[..., n:2 * n]
        ya, yb = turn(a, b, c, sign)
        size = a.abs() + b.abs() + ea + eb
        return (torch.cat([ya, yb, v[..., 2 * n:]], -1),
                torch.cat([ea + eb + size * (ec + 3 * FLOAT)] * 2 + [ev[..., 2 * n:]], -1))
    y, ey = turned(h, eh, False)
    out = {"y": rounded(y, ey, dtype)}
    if g is not None:
        t, et = turned(g, torch.zeros_like(g), True)
        gw = (t * m).reshape(-1, dim)
        egw = (et * m.abs() + t.abs() * em + FLOAT * (t * m).abs()).reshape(-1, dim)
        out["gw"] = rounded(gw.sum(0), egw.sum(0) + (gw.shape[0] + 2) * SUM * gw.abs().sum(0), dtype)
        u, eu = t * wv, et * wv.abs() + FLOAT * (t * wv).abs()
        dot = (u * m).mean(-1, keepdim=True)
        edot = (eu * m.abs() + u.abs() * em).mean(-1, keepdim=True) + (dim + 4) * FLOAT * (u * m).abs().mean(-1, keepdim=True)
        gx = r * (u - m * dot)
        e = r * (eu + em * dot.abs() + m.abs() * edot + 3 * FLOAT * (u.abs() + (m * dot).abs())) + gx.abs() * (0.5 * (dim + 6) + 4) * FLOAT
        out["gx"] = rounded(gx, e, dtype)
    return out


# -------------------------------------------------------------- attention

def in_sight(row, col, window, sinks):
    seen = col[None] <= row[:, None]
    if window is not None:
        seen = seen & ((row[:, None] - col[None] < window) | (col[None] < sinks))
    return seen & (row[:, None] >= 0)


def attention_rows(q, k, v, row, window, sinks, scale, dtype):
    """One head: q [rows, dim] at positions `row` over k, v [keys, dim], float64.  o with its bound, and what the
    backward needs."""
    dim, keys = k.shape[1], k.shape[0]
    seen = in_sight(row, torch.arange(keys, device=k.device), window, sinks)
    z = q @ k.t() * scale
    size = q.abs() @ k.abs().t() * scale
    ez = (dim + 4) * SUM * size
    zs = torch.where(seen, z, -math.inf)
    lse = torch.logsumexp(zs, 1, keepdim=True)
    p = torch.where(seen, torch.exp(zs - torch.where(lse.isinf(), 0.0, lse)), 0.0)
    top = torch.where(seen, z.abs(), 0.0).amax(1, keepdim=True) if keys else z.sum(1, keepdim=True)
    own = ez + 4 * LIB + 8 * FLOAT * top                     # relative, of an exponential
    row_error = (p * own).sum(1, keepdim=True) + (keys + 4) * FLOAT
    u = 0.0 if dtype == torch.float32 else U[dtype]
    # what is below the type's smallest numbers beside a row's largest probability (float16)
    least = 0.0 if dtype == torch.float32 else 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -126
    eo = (p * (own + u)) @ v.abs() + (row_error + u + (keys + 4) * SUM) * (p @ v.abs()) + least * (seen.double() @ v.abs())
    return {"seen": seen, "z": z, "ez": ez, "lse": lse, "p": p, "ep": own + row_error + 8 * FLOAT * lse.abs().nan_to_num(0, 0, 0),
            "o": p @ v, "eo": eo}


def attention(q, k, v, g, window, sinks, scale, lengths, dtype):
    """q, g [batch, tokens, heads, dim], k, v [batch, tokens, groups, dim] in float64 (any device)"""
    batch, tokens, heads, dim = q.shape
    per = heads // k.shape[2]
    scale = dim ** -0.5 if scale is None else scale
    zero = {n: torch.zeros_like(t) for n, t in (("o", q), ("gq", q), ("gk", k), ("gv", k))}
    value, bound = {n: t.clone() for n, t in zero.items()}, {n: t.clone() for n, t in zero.items()}
    lse = torch.full((batch, heads, tokens), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(batch):
        n = tokens if lengths is None else min(max(int(lengths[b]), 0), tokens)
        if n == 0:
            continue
        for h in range(heads):
            j = h // per
            qb, kb, vb = q[b, :n, h], k[b, :n, j], v[b, :n, j]
            r = attention_rows(qb, kb, vb, torch.arange(n, device=q.device), window, sinks, scale, dtype)
            value["o"][b, :n, h], bound["o"][b, :n, h] = rounded(r["o"], r["eo"], dtype)
            lse[b, h, :n] = r["lse"][:, 0]
            if g is None:
                continue
            gb, p, u = g[b, :n, h], r["p"], 0.0 if dtype == torch.float32 else U[dtype]
            dp, d = gb @ vb.t(), (gb * r["o"]).sum(1, keepdim=True)
            edp = (dim + 4) * SUM * (gb.abs() @ vb.abs().t())
            ed = (gb.abs() * bound["o"][b, :n, h]).sum(1, keepdim=True) + (dim + 4) * SUM * (gb * r["o"]).abs().sum(1, keepdim=True)
            ds = p * (dp - d)
            eds = p * (r["ep"] * (dp - d).abs() + edp + ed) * (1 + 2 * u) + u * ds.abs() + 4 * FLOAT * p * (dp.abs() + d.abs())
            # float16 holds ds times a power of two that keeps 2^-24 of what its largest could be, and p times 2^14
            if dtype == torch.float16:
                eds = eds + r["seen"].double() * 2.0 ** -34 * gb.norm(dim=1).max() * vb.norm(dim=1).max()
            epr = p * (r["ep"] + u) + (2.0 ** -39 if dtype == torch.float16 else 0.0) * r["seen"].double()
            # a probability below 2^-126, the smallest normal number, may count as zero: p is off by less than that, ds by
            # that times |dp - d|
            epr, eds = epr + 2.0 ** -126 * r["seen"], eds + 2.0 ** -126 * r["seen"] * (dp.abs() + d.abs())
            for name, a, ea, x, at in (("gq", ds, eds, kb, (b, slice(0, n), h)), ("gk", ds.t(), eds.t(), qb, (b, slice(0, n), j)),
                                       ("gv", p.t(), epr.t(), gb, (b, slice(0, n), j))):
                f = 1.0 if name == "gv" else scale
                value[name][at] += f * (a @ x)
                bound[name][at] += f * (ea @ x.abs() + (per * n + 4) * SUM * (a.abs() @ x.abs()))
    out = {"o": (value["o"], bound["o"]), "lse": lse}
    if g is not None:
        for n in ("gq", "gk", "gv"):
            out[n] = rounded(value[n], bound[n] + 2 * FLOAT * value[n].abs(), dtype)
    return out


def attention_step(q, ck, cv, lengths, window, sinks, scale, dtype):
    batch, tokens, heads, dim = q.shape
    per, capacity = heads // ck.shape[2], ck.shape[1]
    scale = dim ** -0.5 if scale is None else scale
    value, bound = torch.zeros_like(q), torch.zeros_like(q)
    for b in range(batch):
        n = min(max(int(lengths[b]), 0), capacity)
        row = torch.arange(n - tokens, n, device=q.device)
        for h in range(heads):
            r = attention_rows(q[b, :, h], ck[b, :n, h // per], cv[b, :n, h // per], row, window, sinks, scale, dtype)
            value[b, :, h], bound[b, :, h] = rounded(r["o"], r["eo"], dtype)
    return value, bound
