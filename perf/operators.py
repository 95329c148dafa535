"""The classical operators of a hybrid model around ``Circuit``, as measured cases.

  norm    y = (x - mean) / sqrt(var + eps) * weight + bias, over the last axis
  linear  y = act(x W^T + b) + r: features to a circuit's angles, expectations
          back to features with the residual, ordinary projections
  gated   h = act(x Wg^T + bg) * (x Wu^T + bu)

A case's call is

  fwd       the forward call alone (inference)
  step      the forward call, then the backward call (a training step that keeps
            what the forward saved)
  autograd  the same through torch.autograd

``rows`` are samples or tokens, ``inp`` and ``out`` features in and out (a norm
has ``inp`` only), ``stride`` further elements between the rows of x (x is a
slice of a wider tensor).
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_EPS = 1e-5


def _case(name, op, call, dtype, rows, inp, out=0, act="none", bias=True, residual=False, y="", stride=0):
    return {"name": name, "op": op, "call": call, "dtype": dtype, "rows": rows, "inp": inp, "out": out,
            "act": act, "bias": bias, "residual": residual, "y": y or dtype, "stride": stride}


def listed():
    return [
        # the smallest training step of the package's workloads (64 samples): latency and launches only
        _case("norm_step_64x256_f32", "norm", "step", "f32", 64, 256),
        # inference over a batch of prompts: two passes over HBM at most
        _case("norm_fwd_8192x4096_bf16", "norm", "fwd", "bf16", 8192, 4096),
        # training inside a torch model
        _case("norm_autograd_4096x2048_bf16", "norm", "autograd", "bf16", 4096, 2048),
        # odd sizes, rows of a wider tensor
        _case("norm_step_1021x1001_f16", "norm", "step", "f16", 1021, 1001, stride=7),
        # 16-bit features to the float32 angles of a 12-qubit circuit, 4096 samples
        _case("linear_angles_4096x1024to12", "linear", "step", "bf16", 4096, 1024, 12, act="tanh", y="f32"),
        # the float32 expectations of 16 qubits, 512 samples, back to features, with the residual
        _case("linear_features_512x16to1024", "linear", "step", "f32", 512, 16, 1024, residual=True),
        # one token through a projection back to the residual stream: weights are all there is to read
        _case("linear_token_1x4096to4096", "linear", "fwd", "bf16", 1, 4096, 4096, residual=True),
        # odd sizes in every direction, through autograd
        _case("linear_autograd_1023x517to1031", "linear", "autograd", "f16", 1023, 517, 1031, act="silu", residual=True),
        # a projection of a training step: three large products
        _case("linear_step_8192x2048to2048", "linear", "step", "bf16", 8192, 2048, 2048, act="gelu", residual=True),
        # a few tokens through the gated block: its two weights are all there is to read
        _case("gated_token_4x2048to5632", "gated", "fwd", "bf16", 4, 2048, 5632, act="silu", bias=False),
        # a small odd training step through autograd
        _case("gated_autograd_777x504to1365", "gated", "autograd", "f16", 777, 504, 1365, act="gelu"),
        # the largest training step
        _case("gated_step_8192x2048to5632", "gated", "step", "bf16", 8192, 2048, 5632, act="silu", bias=False),
    ]


def _seconds(case):
    """A rough time of a pass, to bound the drawn cases by the listed ones."""
    w = work(case)
    return w["flops"] / 6e13 + w["bytes"] / 1e12


def _size(rng, low, high):
    """Between low and high, even in the logarithm: odd, a power of two, or 5/4 or 7/4 of one."""
    v = 2.0 ** rng.uniform(math.log2(low), math.log2(high))
    kind = rng.randrange(4)
    if kind < 2:
        s = int(v) | 1
    elif kind == 2:
        s = 1 << int(math.log2(v) + 0.5)
    else:
        s = (1 << max(2, int(math.log2(v)))) // 4 * rng.choice((5, 7))
    return min(max(s, low), high)


def draw(rng):
    most = max(_seconds(c) for c in listed())
    while True:
        op = rng.choice(["norm", "linear", "linear", "gated", "gated"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        call = rng.choice(["fwd", "step", "step", "autograd"])
        rows = _size(rng, 1, 16384)
        act = rng.choice(["none", "gelu", "silu", "tanh", "sigmoid"] + (["relu"] if dtype != "f32" else []))
        case = _case("", op, call, dtype, rows, 1, stride=rng.choice((0, 0, 0, 8, 5)))
        del case["name"]
        if op == "norm":
            case["inp"] = _size(rng, 16, 16384)
        elif op == "linear":
            # features to features, features to angles, expectations to features
            kind = rng.choice(["plain", "plain", "angles", "features"])
            case["inp"] = rng.randint(4, 20) if kind == "features" else _size(rng, 32, 8192)
            case["out"] = rng.randint(4, 20) if kind == "angles" else _size(rng, 32, 8192)
            case["act"] = act
            case["residual"] = rng.random() < 0.5
            if kind == "angles" and dtype != "f32":
                case["y"] = "f32"
            if kind == "features" and dtype == "f32":
                case["y"] = rng.choice(["f32", "bf16"])
        else:
            case["inp"], case["out"] = _size(rng, 32, 4096), _size(rng, 32, 8192)
            case["act"] = "silu" if act == "none" else act
        case["bias"] = rng.random() < 0.7
        if _seconds(case) <= most:
            return case


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=None):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype or _DT[case["dtype"]])

    rows, inp, out = case["rows"], case["inp"], case["out"]
    s = dict(case)
    x = torch.randn(rows, inp + case["stride"], generator=g, device="cuda")
    if case["op"] == "norm":
        # a residual stream: rows of different size and offset
        x = x * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda")) \
            + torch.randn(rows, 1, generator=g, device="cuda")
        s["weight"] = (1.0 + 0.2 * torch.randn(inp, generator=g, device="cuda")).to(_DT[case["dtype"]])
        s["bias_"] = normal(inp, scale=0.1) if case["bias"] else None
        s["gy"] = normal(rows, inp)
    elif case["op"] == "linear":
        if inp <= 20:
            x = torch.tanh(x)                      # expectations
        s["weight"] = normal(out, inp, scale=inp ** -0.5)
        s["bias_"] = normal(out, scale=0.1) if case["bias"] else None
        s["res"] = normal(rows, out, dtype=_DT[case["y"]]) if case["residual"] else None
        s["gy"] = normal(rows, out, dtype=_DT[case["y"]])
    else:
        s["weight"], s["up"] = normal(out, inp, scale=inp ** -0.5), normal(out, inp, scale=inp ** -0.5)
        s["bias_"] = normal(out, scale=0.1) if case["bias"] else None
        s["bias_up"] = normal(out, scale=0.1) if case["bias"] else None
        s["gy"] = normal(rows, out)
    s["x"] = x.to(_DT[case["dtype"]])[:, :inp]
    if case["call"] == "autograd":
        s["leaves"] = [t.detach().requires_grad_() for t in
                       (s["x"], s["weight"], s.get("up"), s["bias_"], s.get("bias_up")) if t is not None]
        it = iter(s["leaves"])
        s["x"], s["weight"] = next(it), next(it)
        if case["op"] == "gated":
            s["up"] = next(it)
        if case["bias"]:
            s["bias_"] = next(it)
            if case["op"] == "gated":
                s["bias_up"] = next(it)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2607_11985_gb300 import layers

    op, call, act, x, w, b, gy = s["op"], s["call"], s["act"], s["x"], s["weight"], s["bias_"], s["gy"]
    y_type = _DT[s["y"]]
    if op == "norm":
        if call == "fwd":
            return {"y": layers.layer_norm_forward(x, w, b, _EPS, save=False)}
        if call == "step":
            y, saved = layers.layer_norm_forward(x, w, b, _EPS)
            gx, gw, gb = layers.layer_norm_backward(gy, x, w, saved, need_bias=b is not None)
            return _named(y, gx, gw, gb=gb)
        y = layers.layer_norm(x, w, b, _EPS)
    elif op == "linear":
        if call == "fwd":
            return {"y": layers.linear_forward(x, w, b, act, s["res"], y_type, save=False)}
        if call == "step":
            y, saved = layers.linear_forward(x, w, b, act, s["res"], y_type)
            gx, gw, gb = layers.linear_backward(gy, x, w, saved, act, need_bias=b is not None)
            return _named(y, gx, gw, gb=gb)
        y = layers.linear(x, w, b, act, s["res"], y_type)
    else:
        if call == "fwd":
            return {"y": layers.gated_forward(x, w, s["up"], b, s["bias_up"], act, save=False)}
        if call == "step":
            y, saved = layers.gated_forward(x, w, s["up"], b, s["bias_up"], act)
            gx, gw, gup, gb, gbup = layers.gated_backward(gy, x, w, s["up"], saved, act, need_bias=b is not None)
            return _named(y, gx, gw, gup, gb, gbup)
        y = layers.gated(x, w, s["up"], b, s["bias_up"], act)
    return _of_autograd(s, y, torch.autograd.grad(y, s["leaves"], gy))


def _named(y, gx, gw, gup=None, gb=None, gbup=None):
    return {"y": y, "gx": gx, "gw": gw, "gup": gup, "gb": gb, "gbup": gbup}


def _of_autograd(s, y, grads):
    names = ["gx", "gw"] + ["gup"] * (s["op"] == "gated") + ["gb"] * s["bias"] + ["gbup"] * (s["bias"] and s["op"] == "gated")
    return _named(y.detach(), **dict(zip(names, grads)))


def _act(name, z):
    """act(z) and act'(z) in 32 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        on = (z > 0).float()
        return z * on, on
    if name == "tanh":
        a = torch.tanh(z)
        return a, 1.0 - a * a
    if name == "gelu":                             # z Phi(z), by the error function
        phi = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    p = 1.0 / (1.0 + torch.exp(-z))
    if name == "sigmoid":
        return p, p * (1.0 - p)
    return z * p, p * (1.0 + z * (1.0 - p))         # silu


def _run_plain(s):
    """The same in elementary operations, in 32 bits, each output rounded once."""
    with torch.no_grad():
        dt, grads = _DT[s["dtype"]], s["call"] != "fwd"
        x, w, gy = s["x"].float(), s["weight"].float(), s["gy"].float()
        b = s["bias_"].float() if s["bias"] else 0.0
        if s["op"] == "norm":
            d = x - x.mean(-1, keepdim=True)
            r = torch.rsqrt((d * d).mean(-1, keepdim=True) + _EPS)
            n = d * r
            y = (n * w + b).to(dt)
            if not grads:
                return {"y": y}
            t = gy * w
            gx = r * (t - t.mean(-1, keepdim=True) - n * (t * n).mean(-1, keepdim=True))
            return _named(y, gx.to(dt), (gy * n).sum(0).to(dt), gb=gy.sum(0).to(dt) if s["bias"] else None)
        if s["op"] == "linear":
            a, da = _act(s["act"], x @ w.t() + b)
            y = ((a + s["res"].float()) if s["residual"] else a).to(_DT[s["y"]])
            if not grads:
                return {"y": y}
            dz = gy * da
            return _named(y, (dz @ w).to(dt), (dz.t() @ x).to(dt), gb=dz.sum(0).to(dt) if s["bias"] else None)
        up, bu = s["up"].float(), s["bias_up"].float() if s["bias"] else 0.0
        u = x @ up.t() + bu
        a, da = _act(s["act"], x @ w.t() + b)
        y = (a * u).to(dt)
        if not grads:
            return {"y": y}
        dg, du = gy * u * da, gy * a
        return _named(y, (dg @ w + du @ up).to(dt), (dg.t() @ x).to(dt), (du.t() @ x).to(dt),
                      dg.sum(0).to(dt) if s["bias"] else None, du.sum(0).to(dt) if s["bias"] else None)


# ------------------------------------------------------------------ 64 bits, and the work of a pass

_EXACT = {
    "none": lambda z: z,
    "relu": lambda z: z.clamp(min=0.0),
    "tanh": lambda z: 2.0 / (1.0 + torch.exp(-2.0 * z)) - 1.0,
    "sigmoid": lambda z: 0.5 + 0.5 * torch.tanh(0.5 * z),
    "silu": lambda z: 0.5 * z * (1.0 + torch.tanh(0.5 * z)),
    "gelu": lambda z: 0.5 * z * torch.erfc(-z / math.sqrt(2.0)),
}


def exact(case, seed):
    """The definitions in float64; gradients by differentiating them."""
    if work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    wide = {k: s[k].detach().double() for k in ("x", "weight", "up", "bias_", "bias_up") if s.get(k) is not None}
    leaves = {k: v.requires_grad_(case["call"] != "fwd") for k, v in wide.items()}
    x, w = leaves["x"], leaves["weight"]
    if case["op"] == "norm":
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        y = w * ((x - mean) / torch.sqrt(var + _EPS))
        y = y + leaves["bias_"] if case["bias"] else y
    else:
        z = torch.einsum("tk,nk->tn", x, w)
        y = _EXACT[case["act"]](z + leaves["bias_"] if case["bias"] else z)
        if case["op"] == "gated":
            u = torch.einsum("tk,nk->tn", x, leaves["up"])
            y = y * (u + leaves["bias_up"] if case["bias"] else u)
        elif case["residual"]:
            y = y + s["res"].double()
    if case["call"] == "fwd":
        return {"y": y}
    got = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), s["gy"].double())))
    return _named(y.detach(), got["x"], got["weight"], got.get("up"), got.get("bias_"), got.get("bias_up"))


def work(case):
    """Each input read once, each output written once; the products' operations."""
    size = {"f32": 4, "bf16": 2, "f16": 2}
    rows, inp, out, e, ey = case["rows"], case["inp"], case["out"], size[case["dtype"]], size[case["y"]]
    grads = case["call"] != "fwd"
    if case["op"] == "norm":
        params = (2 if case["bias"] else 1) * inp
        return {"bytes": e * ((4 if grads else 2) * rows * inp + (2 if grads else 1) * params),
                "flops": (20 if grads else 8) * rows * inp}
    two = 2 if case["op"] == "gated" else 1
    weights = two * out * (inp + (1 if case["bias"] else 0))
    ends = (2 if grads else 1) + (1 if case["residual"] else 0)
    return {"bytes": (2 if grads else 1) * e * (rows * inp + weights) + ends * ey * rows * out,
            "flops": two * (6 if grads else 2) * rows * inp * out}
