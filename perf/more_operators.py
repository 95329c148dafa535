"""The operators of a sequence model around ``Circuit``, as measured cases.

  dropout    y = residual + kept * x / (1 - p); element e is kept by word e % 4 of
             Philox 4x32-10 (Salmon et al. 2011) at counter (e / 4, offset), key seed:
             no mask is stored, the backward draws it again
  rotary     queries and keys of each head: x / sqrt(mean(x^2) + eps) * weight, then the
             pairs (i, n + i) turned by position * frequency[i]; the form for serving also
             puts the new keys and values into a cache
  attention  causal, a query at position p sees the last ``window`` positions up to p
             (0: all) and the first ``sinks`` ones; query heads share key heads
  cached     the same for the last tokens of sequences whose keys lie in a cache

A case's call is

  fwd       the forward call alone (inference; the forms for serving have no other)
  step      the forward call, then the backward call (a training step)
  autograd  the same through torch.autograd

``batch`` sequences of ``tokens`` tokens (``cached``: new tokens, in caches of ``capacity``),
``heads`` query and ``groups`` key heads of ``dim`` elements; ``ragged``: sequences of different
lengths, padded; ``stride``: further elements between the tokens of the inputs (heads are slices of
a wider projection).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-6
_BASE = 10000.0


def _dropout(name, call, dtype, rows, cols, p, residual=True):
    return {"name": name, "op": "dropout", "call": call, "dtype": dtype, "rows": rows, "cols": cols, "p": p,
            "residual": residual}


def _rotary(name, call, dtype, batch, tokens, heads, groups, dim, turned=0, stride=0, capacity=0):
    return {"name": name, "op": "rotary", "call": call, "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads,
            "groups": groups, "dim": dim, "turned": turned or dim, "stride": stride, "capacity": capacity}


def _attention(name, call, dtype, batch, tokens, heads, groups, dim, window=0, sinks=0, ragged=False, stride=0):
    return {"name": name, "op": "attention", "call": call, "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads,
            "groups": groups, "dim": dim, "window": window, "sinks": sinks, "ragged": ragged, "stride": stride}


def _cached(name, dtype, batch, tokens, heads, groups, dim, capacity, window=0, sinks=0, ragged=True):
    return {"name": name, "op": "cached", "call": "fwd", "dtype": dtype, "batch": batch, "tokens": tokens, "heads": heads,
            "groups": groups, "dim": dim, "capacity": capacity, "window": window, "sinks": sinks, "ragged": ragged}


def listed():
    return [
        # the smallest training step of the package's workloads (64 samples): latency and launches only
        _dropout("dropout_step_64x256_f32", "step", "f32", 64, 256, 0.1),
        # the residual stream of a large training step
        _dropout("dropout_step_8192x4096_bf16", "step", "bf16", 8192, 4096, 0.1),
        # one new token of each of 16 sequences: queries out, keys and values into the cache
        _rotary("rotary_token_16_bf16", "fwd", "bf16", 16, 1, 32, 8, 128, capacity=512),
        # a training step over four sequences
        _rotary("rotary_step_4x2048_bf16", "step", "bf16", 4, 2048, 32, 8, 128),
        # odd sizes, part of each head turned, heads that are slices of a wider projection
        _rotary("rotary_autograd_3x333_f16", "autograd", "f16", 3, 333, 5, 1, 80, turned=48, stride=24),
        # short float32 sequences of a small hybrid model, through autograd
        _attention("attention_autograd_16x64_f32", "autograd", "f32", 16, 64, 4, 4, 64),
        # odd sizes, a window that ends inside tiles, padded sequences
        _attention("attention_autograd_3x777_f16", "autograd", "f16", 3, 777, 6, 2, 72, window=100, sinks=3, ragged=True, stride=8),
        # a prompt read into a model with a window
        _attention("attention_fwd_2x8192_bf16", "fwd", "bf16", 2, 8192, 16, 4, 128, window=1024, sinks=4),
        # a training step with every earlier position in sight
        _attention("attention_step_4x4096_bf16", "step", "bf16", 4, 4096, 16, 4, 128),
        # the largest training step: one long sequence, a window and its first tokens
        _attention("attention_step_1x32768_bf16", "step", "bf16", 1, 32768, 8, 2, 128, window=4096, sinks=16),
        # a token of one sequence through a window: latency
        _cached("cached_token_1_f16", "f16", 1, 1, 16, 2, 64, 1999, window=512, sinks=4, ragged=False),
        # a token of each of 24 sequences, every cached position in sight: the cache is all there is to read
        _cached("cached_token_24_bf16", "bf16", 24, 1, 32, 8, 128, 8192),
    ]


def _lengths(case):
    """Tokens of each sequence: from all down to a third."""
    most, batch = case.get("capacity") or case["tokens"], case["batch"]
    return [max(most - (2 * most * b // (3 * batch) if case["ragged"] else 0), min(most, case["tokens"]) if case["op"] == "cached" else 1)
            for b in range(batch)]


def _size(rng, low, high):
    """Between low and high, even in the logarithm: odd, or a power of two, or 5/4 or 7/4 of one."""
    v = 2.0 ** rng.uniform(math.log2(low), math.log2(high))
    kind = rng.randrange(4)
    if kind < 2:
        s = int(v) | 1
    elif kind == 2:
        s = 1 << int(math.log2(v) + 0.5)
    else:
        s = (1 << max(2, int(math.log2(v)))) // 4 * rng.choice((5, 7))
    return min(max(s, low), high)


def _seconds(case):
    """A rough time of a pass in elementary operations, to bound the drawn cases by the listed ones."""
    w = work(case)
    return w["flops"] / 3e13 + w["bytes"] / 1e12


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        op = rng.choice(["dropout", "rotary", "attention", "attention", "cached"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        call = rng.choice(["fwd", "step", "step", "autograd"])
        groups = rng.choice((1, 2, 4, 8))
        heads = groups * rng.choice((1, 1, 2, 3, 4, 8))
        dim = rng.choice((16, 32, 40, 64, 64, 72, 80, 96, 128, 128))
        window = rng.choice((0, _size(rng, 16, 4096)))
        sinks = rng.choice((0, 1, 4, 16)) if window else 0
        stride = rng.choice((0, 0, 8, 5))
        if op == "dropout":
            case = _dropout("", call, dtype, _size(rng, 1, 16384), _size(rng, 16, 8192), rng.choice((0.05, 0.1, 0.5)), rng.random() < 0.5)
        elif op == "rotary":
            turned = rng.choice((dim, dim, dim // 2))
            if rng.random() < 0.3:
                case = _rotary("", "fwd", dtype, _size(rng, 1, 64), rng.choice((1, 1, 3)), heads, groups, dim, turned, stride, 256)
            else:
                case = _rotary("", call, dtype, rng.choice((1, 2, 3, 8)), _size(rng, 1, 8192), heads, groups, dim, turned, stride)
        elif op == "attention":
            case = _attention("", call, dtype, rng.choice((1, 2, 3, 8)), _size(rng, 1, 16384), heads, groups, dim, window, sinks,
                              rng.random() < 0.3, stride)
            if dtype == "f32" and case["tokens"] > 2048:
                continue
        else:
            case = _cached("", dtype, _size(rng, 1, 64), rng.choice((1, 1, 1, 2, 4)), heads, groups, dim, _size(rng, 64, 65536), window, sinks,
                           rng.random() < 0.7)
            if work(dict(case, window=0))["bytes"] > 4e9:        # caches of a few GB
                continue
        del case["name"]
        if _seconds(case) <= most:
            return case


# ------------------------------------------------------------------ inputs

def _frequencies(case):
    n = case["turned"] // 2
    return torch.tensor([_BASE ** (-i / n) for i in range(n)], dtype=torch.float64, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _DT[case["dtype"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    s = dict(case)
    if case["op"] == "dropout":
        shape = (case["rows"], case["cols"])
        s["x"], s["gy"] = normal(*shape), normal(*shape)
        s["res"] = normal(*shape) if case["residual"] else None
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ seed, seed % 1000      # of a run, of a layer and step
        leaves = ["x", "res"] if case["residual"] else ["x"]
    else:
        batch, tokens, dim = case["batch"], case["tokens"], case["dim"]

        def rows(heads):
            wide = normal(batch, tokens, heads * dim + case.get("stride", 0))
            return wide[..., :heads * dim].unflatten(-1, (heads, dim))

        s["q"] = rows(case["heads"])
        if case["op"] != "cached":
            s["k"] = rows(case["groups"])
        if case["op"] == "rotary":
            s["wq"], s["wk"] = (1.0 + 0.2 * normal(dim)), (1.0 + 0.2 * normal(dim))
            s["freq"] = _frequencies(case)
            if case["capacity"]:
                s["v"] = rows(case["groups"])
                s["ck"], s["cv"] = (normal(batch, case["capacity"], case["groups"], dim) for _ in range(2))
                s["lengths"] = torch.randint(tokens, case["capacity"] + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)
            else:
                # sequences that begin anywhere in a long text
                start = torch.randint(0, 100000, (batch, 1), generator=g, device="cuda", dtype=torch.int32)
                s["positions"] = start + torch.arange(tokens, device="cuda", dtype=torch.int32)
                s["gq"], s["gk"] = normal(batch, tokens, case["heads"], dim), normal(batch, tokens, case["groups"], dim)
            leaves = ["q", "k", "wq", "wk"]
        else:
            s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] or case["op"] == "cached" else None
            if case["op"] == "attention":
                s["v"] = rows(case["groups"])
                s["go"] = normal(batch, tokens, case["heads"], dim)
            else:
                s["ck"], s["cv"] = (normal(batch, case["capacity"], case["groups"], dim) for _ in range(2))
            leaves = ["q", "k", "v"]
    if case["call"] == "autograd":
        for n in leaves:
            s[n] = s[n].detach().requires_grad_()
        s["leaves"] = [s[n] for n in leaves]
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2607_11985_gb300 import layers

    op, call = s["op"], s["call"]
    if op == "dropout":
        a = (s["p"], s["seed"], s["offset"])
        if call == "autograd":
            y = layers.dropout(s["x"], *a, s["res"])
            grads = torch.autograd.grad(y, s["leaves"], s["gy"])
            return {"y": y.detach(), "gx": grads[0], "gr": grads[1] if s["residual"] else None}
        y = layers.dropout_forward(s["x"], *a, s["res"])
        if call == "fwd":
            return {"y": y}
        return {"y": y, "gx": layers.dropout_backward(s["gy"], *a), "gr": s["gy"] if s["residual"] else None}
    if op == "rotary":
        w = (s["wq"], s["wk"], s["freq"])
        if s["capacity"]:
            q = layers.norm_rotary_step(s["q"], s["k"], s["v"], s["ck"], s["cv"], s["lengths"], *w, _EPS)
            return {"q": q, "ck": s["ck"], "cv": s["cv"]}
        w += (s["positions"], _EPS)
        if call == "autograd":
            q, k = layers.norm_rotary(s["q"], s["k"], *w)
            grads = torch.autograd.grad((q, k), s["leaves"], (s["gq"], s["gk"]))
            return dict(zip(("q", "k", "gq", "gk", "gwq", "gwk"), (q.detach(), k.detach(), *grads)))
        q, k = layers.norm_rotary_forward(s["q"], s["k"], *w)
        if call == "fwd":
            return {"q": q, "k": k}
        return dict(zip(("q", "k", "gq", "gk", "gwq", "gwk"), (q, k, *layers.norm_rotary_backward(s["gq"], s["gk"], s["q"], s["k"], *w))))
    sight = {"window": s["window"] or None, "sinks": s["sinks"]}
    if op == "cached":
        return {"o": layers.attention_step(s["q"], s["ck"], s["cv"], s["lengths"], **sight)}
    sight["lengths"] = s["lengths"]
    q, k, v = s["q"], s["k"], s["v"]
    if call == "fwd":
        return {"o": layers.attention_forward(q, k, v, save=False, **sight)}
    if call == "step":
        o, saved = layers.attention_forward(q, k, v, **sight)
        grads = layers.attention_backward(s["go"], q, k, v, o, saved, **sight)
    else:
        o = layers.attention(q, k, v, **sight)
        grads = torch.autograd.grad(o, s["leaves"], s["go"])
    return dict(zip(("o", "gq", "gk", "gv"), (o.detach(), *grads)))


def _words(groups, offset, seed, device):
    """Philox 4x32-10: four 32-bit words for each counter (e, offset), in 64-bit integers."""
    low = 0xFFFFFFFF
    c = [groups & low, groups >> 32, torch.full_like(groups, offset & low), torch.full_like(groups, offset >> 32)]
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57       # modulo 2^64, as two's complement
        c = [(b >> 32 & low) ^ c[1] ^ k0, b & low, (a >> 32 & low) ^ c[3] ^ k1, a & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(c, -1)


def _run_plain(s):
    """The same in elementary operations, in 32 bits, each output rounded once."""
    with torch.no_grad():
        if s["op"] == "dropout":
            return _plain_dropout(s)
        if s["op"] == "rotary":
            return _plain_rotary(s)
        return _plain_cached(s) if s["op"] == "cached" else _plain_attention(s)


def _plain_dropout(s):
    dt, x = _DT[s["dtype"]], s["x"].float()
    n = x.numel()
    words = _words(torch.arange((n + 3) // 4, device=x.device), s["offset"], s["seed"], x.device).reshape(-1)[:n].reshape(x.shape)
    factor = (words >= round(s["p"] * 2 ** 32)).float() * (1.0 / (1.0 - s["p"]))
    y = x * factor
    y = (y + s["res"].float() if s["residual"] else y).to(dt)
    if s["call"] == "fwd":
        return {"y": y}
    return {"y": y, "gx": (s["gy"].float() * factor).to(dt), "gr": s["gy"] if s["residual"] else None}


def _turn(x, c, d):
    """The pairs (i, n + i) of the last axis turned; columns from 2n on stay."""
    n = c.shape[-1]
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * c - b * d, b * c + a * d, x[..., 2 * n:]], -1)


def _plain_rotary(s):
    dt = _DT[s["dtype"]]
    if s["capacity"]:
        pos = (s["lengths"].long() - s["tokens"])[:, None] + torch.arange(s["tokens"], device="cuda")
    else:
        pos = s["positions"]
    angle = (pos.double()[..., None] * s["freq"])[:, :, None]
    c, d = torch.cos(angle).float(), torch.sin(angle).float()
    y, back = [], []
    for x, w, g in ((s["q"], s["wq"], s.get("gq")), (s["k"], s["wk"], s.get("gk"))):
        x, w = x.float(), w.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
        h = x * r
        y.append(_turn(h * w, c, d).to(dt))
        if s["call"] != "fwd":
            t = _turn(g.float(), c, -d)
            u = t * w
            back.append(((r * (u - h * (u * h).mean(-1, keepdim=True))).to(dt), (t * h).sum((0, 1, 2)).to(dt)))
    if s["capacity"]:
        at = torch.arange(s["batch"], device="cuda")[:, None]
        s["ck"][at, pos] = y[1]
        s["cv"][at, pos] = s["v"]
        return {"q": y[0], "ck": s["ck"], "cv": s["cv"]}
    if s["call"] == "fwd":
        return {"q": y[0], "k": y[1]}
    return {"q": y[0], "k": y[1], "gq": back[0][0], "gk": back[1][0], "gwq": back[0][1], "gwk": back[1][1]}


def _heads_first(x, groups):
    """[batch, tokens, heads, dim] as [batch, groups, heads of a group * tokens, dim] in 32 bits"""
    b, t, h, d = x.shape
    return x.float().permute(0, 2, 1, 3).reshape(b, groups, h // groups * t, d)


def _tokens_first(x, heads, tokens):
    b, _, _, d = x.shape
    return x.reshape(b, heads, tokens, d).permute(0, 2, 1, 3)


def _plain_attention(s):
    """In blocks of queries, each with the keys that one of them may see."""
    dt, batch, n, heads, groups, dim = _DT[s["dtype"]], s["batch"], s["tokens"], s["heads"], s["groups"], s["dim"]
    scale, window = dim ** -0.5, s["window"] or n
    k, v = _heads_first(s["k"], groups), _heads_first(s["v"], groups)
    grads = s["call"] != "fwd"
    length = s["lengths"] if s["lengths"] is not None else torch.full((batch,), n, device="cuda")
    o_all, gq_all = [], []
    gk, gv = torch.zeros_like(k), torch.zeros_like(v)
    for q0 in range(0, n, 1024):
        q1 = min(n, q0 + 1024)
        first = max(0, q0 - window + 1)
        sink = min(s["sinks"], first)
        at = torch.cat([torch.arange(sink, device="cuda"), torch.arange(first, q1, device="cuda")])
        row = torch.arange(q0, q1, device="cuda")
        seen = (at <= row[:, None]) & ((at > row[:, None] - window) | (at < s["sinks"])) & (row[:, None] < length[:, None, None])
        seen = seen[:, None, None]                                        # [batch, 1, 1, rows, keys]
        q = _heads_first(s["q"][:, q0:q1], groups)
        kb, vb = (torch.cat([x[:, :, :sink], x[:, :, first:q1]], 2) for x in (k, v))
        shape = (batch, groups, heads // groups, q1 - q0, len(at))
        z = ((q @ kb.transpose(2, 3)) * scale).reshape(shape).masked_fill(~seen, -math.inf)
        z = torch.exp(z - z.amax(-1, keepdim=True).clamp(min=-1e30))      # rows that see nothing: zeros
        total = z.sum(-1, keepdim=True)
        p = (z / torch.where(total > 0, total, 1.0)).reshape(batch, groups, -1, len(at))
        o = p @ vb
        o_all.append(_tokens_first(o, heads, q1 - q0))
        if grads:
            go = _heads_first(s["go"][:, q0:q1], groups)
            ds = p * (go @ vb.transpose(2, 3) - (go * o).sum(-1, keepdim=True)) * scale
            gq_all.append(_tokens_first(ds @ kb, heads, q1 - q0))
            for total, part in ((gk, ds.transpose(2, 3) @ q), (gv, p.transpose(2, 3) @ go)):
                total[:, :, :sink] += part[:, :, :sink]
                total[:, :, first:q1] += part[:, :, sink:]
    o = torch.cat(o_all, 1).to(dt)
    if not grads:
        return {"o": o}
    return {"o": o, "gq": torch.cat(gq_all, 1).to(dt), "gk": _tokens_first(gk, groups, n).to(dt), "gv": _tokens_first(gv, groups, n).to(dt)}


def _plain_cached(s):
    dt, batch, n, heads, groups, dim, m = (_DT[s["dtype"]], s["batch"], s["tokens"], s["heads"], s["groups"], s["dim"], s["capacity"])
    row = (s["lengths"] - n)[:, None, None] + torch.arange(n, device="cuda")[:, None]
    at = torch.arange(m, device="cuda")
    seen = ((at <= row) & ((at > row - (s["window"] or m)) | (at < s["sinks"])))[:, None, None]
    q, k, v = (_heads_first(x, groups) for x in (s["q"], s["ck"], s["cv"]))
    z = ((q @ k.transpose(2, 3)) * dim ** -0.5).reshape(batch, groups, heads // groups, n, m).masked_fill(~seen, -math.inf)
    z = torch.exp(z - z.amax(-1, keepdim=True))
    p = (z / z.sum(-1, keepdim=True)).reshape(batch, groups, -1, m)
    return {"o": _tokens_first(p @ v, heads, n).to(dt)}


# ------------------------------------------------------------------ 64 bits, and the work of a pass

def exact(case, seed):
    """The definitions in float64; gradients by differentiating them."""
    s = prepare(case, seed)
    return {"dropout": _exact_dropout, "rotary": _exact_rotary, "attention": _exact_attention, "cached": _exact_cached}[case["op"]](s)


def _exact_dropout(s):
    n = s["rows"] * s["cols"]
    e = np.arange((n + 3) // 4, dtype=np.uint64)
    m, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = np.stack([e & m, e >> half, np.full_like(e, s["offset"] & 0xFFFFFFFF), np.full_like(e, s["offset"] >> 32)])
    for r in range(10):
        k0 = np.uint64(((s["seed"] & 0xFFFFFFFF) + r * 0x9E3779B9) & 0xFFFFFFFF)
        k1 = np.uint64(((s["seed"] >> 32) + r * 0xBB67AE85) & 0xFFFFFFFF)
        first, second = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = np.stack([(second >> half) ^ c[1] ^ k0, second & m, (first >> half) ^ c[3] ^ k1, first & m])
    kept = torch.from_numpy((c.T.reshape(-1)[:n] >= np.uint64(round(s["p"] * 2 ** 32))).reshape(s["rows"], s["cols"])).cuda()
    x, res, gy = (None if s[k] is None else s[k].detach().double() for k in ("x", "res", "gy"))
    y = torch.where(kept, x / (1.0 - s["p"]), 0.0)
    y = y + res if res is not None else y
    if s["call"] == "fwd":
        return {"y": y}
    return {"y": y, "gx": torch.where(kept, gy / (1.0 - s["p"]), 0.0), "gr": gy if res is not None else None}


def _exact_rotary(s):
    grads = s["call"] != "fwd"
    q, k, wq, wk = (s[n].detach().double().requires_grad_(grads) for n in ("q", "k", "wq", "wk"))
    if s["capacity"]:
        pos = torch.stack([torch.arange(int(n) - s["tokens"], int(n), device="cuda") for n in s["lengths"]])
    else:
        pos = s["positions"]
    n = s["turned"] // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.einsum("bt,n->btn", pos.double(), s["freq"]))[:, :, None]
    y = []
    for x, w in ((q, wq), (k, wk)):
        h = w * x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS)
        z = torch.complex(h[..., :n], h[..., n:2 * n]) * turn
        y.append(torch.cat([z.real, z.imag, h[..., 2 * n:]], -1))
    if s["capacity"]:
        ck, cv = s["ck"].double(), s["cv"].double()
        for b in range(s["batch"]):
            ck[b, pos[b]], cv[b, pos[b]] = y[1][b], s["v"][b].double()
        return {"q": y[0], "ck": ck, "cv": cv}
    if not grads:
        return {"q": y[0], "k": y[1]}
    g = torch.autograd.grad(y, (q, k, wq, wk), (s["gq"].double(), s["gk"].double()))
    return dict(zip(("q", "k", "gq", "gk", "gwq", "gwk"), (y[0].detach(), y[1].detach(), *g)))


def _exact_rows(q, k, v, row, s):
    """softmax over the keys in sight of the queries q [rows, dim] at positions row, times v"""
    at = torch.arange(k.shape[0], device="cuda")
    seen = at[None] <= row[:, None]
    if s["window"]:
        seen = seen & ((row[:, None] - at[None] < s["window"]) | (at[None] < s["sinks"]))
    used = seen.any(0).nonzero()[:, 0]
    z = torch.einsum("td,kd->tk", q, k[used]) / math.sqrt(s["dim"])
    return torch.softmax(torch.where(seen[:, used], z, -math.inf), 1) @ v[used]


def _exact_attention(s):
    if 2 * work(s)["flops"] > 8e12:
        return None
    grads = s["call"] != "fwd"
    per = s["heads"] // s["groups"]
    q, k, v = (s[n].detach().double() for n in ("q", "k", "v"))
    o, gq, gk, gv = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, q, k, v))
    for b, n in enumerate(_lengths(s)):
        for h in range(s["heads"]):
            kb, vb = (x[b, :n, h // per].clone().requires_grad_(grads) for x in (k, v))
            for q0 in range(0, n, 2048):
                rows = slice(q0, min(n, q0 + 2048))
                qb = q[b, rows, h].clone().requires_grad_(grads)
                y = _exact_rows(qb, kb[:rows.stop], vb[:rows.stop], torch.arange(q0, rows.stop, device="cuda"), s)
                o[b, rows, h] = y.detach()
                if grads:
                    a, c, d = torch.autograd.grad(y, (qb, kb, vb), s["go"][b, rows, h].double())
                    gq[b, rows, h] = a
                    gk[b, :n, h // per] += c
                    gv[b, :n, h // per] += d
    return {"o": o, "gq": gq, "gk": gk, "gv": gv} if grads else {"o": o}


def _exact_cached(s):
    per = s["heads"] // s["groups"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(s)):
        row = torch.arange(n - s["tokens"], n, device="cuda")
        for j in range(s["groups"]):
            k, v = s["ck"][b, :n, j].double(), s["cv"][b, :n, j].double()
            for h in range(j * per, (j + 1) * per):
                o[b, :, h] = _exact_rows(s["q"][b, :, h].double(), k, v, row, s)
    return {"o": o}


def _pairs(first, last, window, sinks):
    """(query, key) pairs of the queries at positions first to last - 1, and the keys that one of them sees"""
    p = np.arange(first, last, dtype=np.int64) + 1
    seen = np.minimum(p, window) + np.minimum(np.maximum(p - window, 0), sinks) if window else p
    low = max(0, first + 1 - window) if window else 0
    return int(seen.sum()), last - low + min(sinks, low)


def work(case):
    """Each input read once, each output written once; two operations for each product and sum."""
    e, grads = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]], case["call"] != "fwd"
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": e * n * ((4 if grads else 2) + (1 if case["residual"] else 0)), "flops": n * (4 if grads else 2)}
    batch, tokens, heads, groups, dim = (case[k] for k in ("batch", "tokens", "heads", "groups", "dim"))
    ends = tokens * batch * dim * e
    if case["op"] == "rotary":
        n = ends * (heads + groups)
        more = 2 * ends * groups if case["capacity"] else 0
        return {"bytes": (4 if grads else 2) * n + more + 2 * dim * e, "flops": n // e * (20 if grads else 8)}
    counts = [_pairs(max(0, n - tokens) if case["op"] == "cached" else 0, n, case["window"], case["sinks"]) for n in _lengths(case)]
    flops = 4 * dim * heads * sum(c[0] for c in counts)
    if case["op"] == "cached":
        return {"bytes": 2 * ends * heads + 2 * groups * dim * e * sum(c[1] for c in counts), "flops": flops}
    return {"bytes": (2 if grads else 1) * 2 * ends * (heads + groups), "flops": flops // 2 * 7 if grads else flops}
