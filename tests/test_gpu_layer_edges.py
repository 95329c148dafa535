"""Layer operators at the edges: of their types' range and bits, of torch's views, tangents
and devices, and of the time that they may take.
"""

import json
import math
import os
import subprocess
import sys
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DIGITS = {F32: 24, BF16: 8, F16: 11}                 # significant bits of a type
LEAST = {F32: -149, BF16: -133, F16: -24}            # exponent of its smallest number


@pytest.fixture(scope="module", autouse=True)
def cuda_ready():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


@pytest.fixture(scope="module")
def layers():
    from paper_2607_11985_gb300 import layers
    return layers


def sync():
    from paper_2607_11985_gb300 import binding
    binding.vqc_sync_check(torch.cuda.current_stream().cuda_stream)


def normal(seed, *shape, scale=1.0, dtype=F32):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype)


def half_unit(v, dtype):
    """The largest error of rounding the float64 values v to dtype once."""
    _, e = torch.frexp(v)
    return torch.ldexp(torch.ones_like(v), (e - DIGITS[dtype]).clamp(min=LEAST[dtype]) - 1)


def sum_error(a, b):
    """a @ b in float sums that may cut: 2^-23 of the magnitudes for each of their
    terms, two for the sum of parts."""
    return (a.shape[1] + 2) * 2.0 ** -23 * (a.abs() @ b.abs())


def once(got, a, b, dtype, what, more=0.0):
    """got is a @ b in float sums, rounded once."""
    want = a @ b
    e = sum_error(a, b) + more
    d = (got.double().cpu() - want).abs()
    bound = half_unit(want.abs() + e, dtype) + e
    assert bool((d <= bound).all()), "%s: %d of %d outside, worst %g of the bound" % (
        what, int((d > bound).sum()), d.numel(), float((d / bound).max()))


def same_infinities(got, want, what):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    there = torch.isinf(want)
    assert bool(there.any()) and torch.equal(got[there], want[there]), what
    assert bool(torch.isfinite(got[torch.isfinite(want)]).all()), what


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(512, 1024, 4), (8, 1000, 600)])
def test_gradients_of_float_outputs_round_once(layers, dtype, rows, inp, out):
    """dz is grad_y itself here, a float32 matrix: the gradients are its products in float
    sums, rounded once.  dz is held in two parts, to 2^-16 in bfloat16 (the first is cut to 8 bits, the
    second rounded to 8) and to 2^-22 in float16."""
    x, w, gy = normal(1, rows, inp, dtype=dtype), normal(2, out, inp, dtype=dtype), normal(3, rows, out)
    gx, gw, _ = layers.linear_backward(gy.cuda(), x.cuda(), w.cuda(), None, "none")
    sync()
    held = 2.0 ** (-16 if dtype == BF16 else -22)
    for got, a, b in ((gx, gy.double(), w.double()), (gw, gy.double().t(), x.double())):
        once(got, a, b, dtype, "gradient", held * (a.abs() @ b.abs()))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(40, 24, 16), (2048, 1024, 1024)])
def test_infinite_weights_and_features_in_gradients(layers, dtype, rows, inp, out):
    """An infinite weight makes the gradients that it enters infinite, of the sign of dz
    times its own, or NaN where dz is zero, in both sizes of a backward; so does an
    infinite feature."""
    x, w, gy = normal(1, rows, inp, dtype=dtype), normal(2, out, inp, dtype=dtype), normal(3, rows, out)
    gy[0, 3], gy[1, 3], gy[2, 3], gy[3, 3], gy[4, 3] = 0.5, 0.0, 1.0, -2.0, 0.3
    w[3, 5], w[3, 6], x[2, 7], x[4, 8] = math.inf, -math.inf, math.inf, -math.inf
    gx, gw, _ = layers.linear_backward(gy.cuda(), x.cuda(), w.cuda(), None, "none")
    sync()
    same_infinities(gx, gy.double() @ w.double(), "gx")
    same_infinities(gw, gy.double().t() @ x.double(), "gw")


@pytest.mark.parametrize("scale", [1e-7, 1e5])
@pytest.mark.parametrize("rows,inp,out", [(4096, 64, 12), (2048, 1024, 1024)])
def test_float16_gradients_of_small_and_large_dz(layers, scale, rows, inp, out):
    """dz outside of float16's range, its gradients inside: the sums of many small terms,
    the products of large ones with small weights.  Above 6e9 operations dz is rounded to
    11 bits, 2^-11 of each term; what is below 2^-38 of the largest may be lost."""
    toward = 1.0 if scale < 1 else 1e-5
    x, w = normal(1, rows, inp, scale=toward, dtype=F16), normal(2, out, inp, scale=toward, dtype=F16)
    gy = normal(3, rows, out, scale=scale)
    gx, gw, _ = layers.linear_backward(gy.cuda(), x.cuda(), w.cuda(), None, "none")
    sync()
    rounding = 2.0 ** -11 if 4.0 * rows * inp * out > 6e9 else 0.0
    for got, a, b in ((gx, gy.double(), w.double()), (gw, gy.double().t(), x.double())):
        lost = 2.0 ** -38 * gy.abs().max().double() * b.abs().sum(0, keepdim=True)
        once(got, a, b, F16, "scale %g" % scale, lost + rounding * (a.abs() @ b.abs()))


def test_float16_gate_of_small_gradients(layers):
    """dg = grad_h u act'(g) and du = grad_h act(g) of a grad_h near float16's smallest
    numbers: bits of dg and du below those numbers count in sums over many rows.
    Bound: the forward's g and u are known to 2^-20 of their terms (depth 32), silu and
    its slope to 2^-20; three roundings of dg, float sums, one rounding."""
    rows, inp, out = 4096, 32, 16
    x, wg, wu = normal(1, rows, inp, dtype=F16), normal(2, out, inp, scale=0.1, dtype=F16), normal(3, out, inp, scale=0.1, dtype=F16)
    gh = normal(4, rows, out, scale=1e-6).to(F16)
    X, WG, WU = x.cuda(), wg.cuda(), wu.cuda()
    _, saved = layers.gated_forward(X, WG, WU)
    gx, gwg, gwu, _, _ = layers.gated_backward(gh.cuda(), X, WG, WU, saved, need_bias=False)
    sync()
    g, u = saved.cpu().double()
    p = torch.sigmoid(g)
    dg, du = gh.double() * u * p * (1 + g * (1 - p)), gh.double() * g * p
    for got, d in ((gwg, dg), (gwu, du)):
        once(got, d.t(), x.double(), F16, "gw", 2.0 ** -18 * (d.t().abs() @ x.double().abs()) +
             2.0 ** -38 * float(d.abs().max()) * x.double().abs().sum(0, keepdim=True) +
             2.0 ** -20 * (gh.double().abs().t() @ x.double().abs()))
    both, wide = torch.cat([dg, du], 1), torch.cat([wg, wu], 0).double()
    once(gx, both, wide, F16, "gx", 2.0 ** -18 * (both.abs() @ wide.abs()) + 2.0 ** -38 * float(both.abs().max()) * wide.abs().sum(0, keepdim=True)
         + 2.0 ** -20 * (torch.cat([gh, gh], 1).double().abs() @ wide.abs()))


def milliseconds(f):
    for _ in range(3):
        f()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    start.record()
    for _ in range(5):
        f()
    end.record()
    torch.cuda.synchronize()
    return start.elapsed_time(end) / 5


def test_float_products_of_values_that_are_not_finite_take_no_longer(layers):
    """A NaN in one weight row, and a model that is NaN throughout: the work of a product does
    not depend on its values (tenfold for what a clock may move)."""
    x, w = normal(1, 1024, 1024).cuda(), normal(2, 1024, 1024).cuda()
    clean = milliseconds(lambda: layers.linear_forward(x, w, save=False))
    w[17] = math.nan
    row = milliseconds(lambda: layers.linear_forward(x, w, save=False))
    y = layers.linear_forward(x, w, save=False)
    assert bool(torch.isnan(y[:, 17]).all()) and int(torch.isnan(y).sum()) == 1024
    w[:] = math.inf
    x[:] = -1.0
    full = milliseconds(lambda: layers.linear_forward(x, w, save=False))
    assert bool((layers.linear_forward(x, w, save=False) == -math.inf).all())
    sync()
    assert max(row, full) <= 10 * clean, (clean, row, full)


def test_float_parts_of_infinite_and_zero_operands(layers):
    """Infinite against infinite, zero, positive and negative operands on both sides of a
    float product in parts, and sums that leave the range."""
    rows, inp, out = 800, 640, 800
    x, w, gy = normal(1, rows, inp), normal(2, out, inp), normal(3, rows, out)
    x[0, 0], x[1, 0], x[2, 1], x[3, 2] = math.inf, -math.inf, math.nan, math.inf
    w[0, 0], w[1, 0], w[2, 0], w[3, 5], w[4, 2], w[5, 2] = math.inf, -math.inf, 0.0, math.nan, 0.0, -1e-30
    gy[6, 0], gy[6, 1], gy[7, 0], gy[8, 9], gy[10, 11] = 0.0, 2.0, math.inf, -math.inf, 1e-30
    x[9], w[9] = 1e30, 1e30
    y = layers.linear_forward(x.cuda(), w.cuda(), save=False)
    gx, gw, _ = layers.linear_backward(gy.cuda(), x.cuda(), w.cuda(), None, "none")
    sync()
    for got, a, b in ((y, x, w.t()), (gx, gy, w), (gw, gy.t(), x)):
        want = a.double() @ b.double()
        same_infinities(got, torch.where(want.abs() > 3.4028235677973366e38, torch.sign(want) * math.inf, want), got.shape)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows", [2, 8, 16])
def test_float_outputs_of_few_rows_and_deep_contractions(layers, dtype, rows):
    """A float32 output keeps a float32 sum's accuracy with few rows as well.  All terms
    positive, so that cuts add up: at most 2^-23 of a chunk's sum at each of its 16 products,
    half of that on average (16 * 2^-24), and 32 roundings of the sum of chunks
    (32 * 2^-25)."""
    inp, out = 8192, 20000
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (0.5 + torch.rand(rows, inp, generator=g, device="cuda")).to(dtype)
    w = (0.5 + torch.rand(out, inp, generator=g, device="cuda")).to(dtype)
    y = layers.linear_forward(x, w, None, "none", out_dtype=F32, save=False)
    sync()
    want = torch.cat([x.double() @ w[i:i + 4000].double().t() for i in range(0, out, 4000)], 1)
    assert float((y.double() - want).norm() / want.norm()) <= 16 * 2.0 ** -24 + 32 * 2.0 ** -25


def test_gelu_in_float_over_its_range(layers):
    """z Phi(z) and its derivative to 2^-20 of their terms, as functions of the math library
    are: the tail as well, where Phi itself is small."""
    z = torch.cat([torch.linspace(-12.5, 12.5, 40001), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 1e19, -1e19])])
    x, one = z[:, None].cuda(), torch.ones(1, 1, device="cuda")
    y, saved = layers.linear_forward(x, one, None, "gelu")
    gx, _, _ = layers.linear_backward(torch.ones_like(y), x, one, saved, "gelu", need_weight=False, need_bias=False)
    sync()
    assert torch.equal(saved.cpu()[:, 0], z)
    v = z.double()
    phi, pdf = 0.5 * torch.erfc(-v / math.sqrt(2.0)), torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    tiny = 2.0 ** -126
    d = (y[:, 0].double().cpu() - v * phi).abs() / (2.0 ** -20 * (v * phi).abs() + tiny)
    assert float(d.max()) <= 1, (float(d.max()), float(v[d.argmax()]))
    d = (gx[:, 0].double().cpu() - phi - v * pdf).abs() / (2.0 ** -20 * (phi + (v * pdf).abs()) + tiny)
    assert float(d.max()) <= 1, (float(d.max()), float(v[d.argmax()]))


@pytest.mark.parametrize("which", ["layer_norm", "linear", "gated"])
def test_tangents_are_refused(layers, which):
    """Forward-mode derivatives are not there: refused, not dropped, for every input, for
    inputs that need a gradient as well, and for an incoming gradient."""
    import torch.autograd.forward_ad as fwd
    x, w, u, b, c, r, nw, nb = (normal(i, *s).cuda() for i, s in
                                enumerate([(6, 8), (5, 8), (5, 8), (5,), (5,), (6, 5), (8,), (8,)]))
    f, ops = {"layer_norm": (layers.layer_norm, [x, nw, nb]),
              "linear": (lambda x, w, b, r: layers.linear(x, w, b, "tanh", r), [x, w, b, r]),
              "gated": (layers.gated, [x, w, u, b, c])}[which]
    for i in range(len(ops)):
        for needs in (False, True):
            with fwd.dual_level():
                some = [t.clone().requires_grad_(needs) for t in ops]
                some[i] = fwd.make_dual(some[i], torch.ones_like(some[i]))
                with pytest.raises(RuntimeError, match="[Ff]orward"):
                    f(*some)
                with torch.no_grad(), pytest.raises(RuntimeError, match="[Ff]orward"):
                    f(*some)
    leaves = [t.clone().requires_grad_() for t in ops]
    y = f(*leaves)
    with fwd.dual_level():
        gy = fwd.make_dual(torch.ones_like(y), torch.ones_like(y))
        for graph in (False, True):
            with pytest.raises(RuntimeError, match="[Ff]orward"):
                torch.autograd.grad(y, leaves, gy, retain_graph=True, create_graph=graph)
    torch.autograd.grad(y, leaves, torch.ones_like(y))
    sync()


def test_residual_of_other_leading_axes(layers):
    """A residual with as many rows as x in other leading axes: its gradient has its shape."""
    x, w = normal(1, 3, 5, 8).cuda().requires_grad_(), normal(2, 6, 8).cuda().requires_grad_()
    for shape in ((15, 6), (5, 3, 6), (1, 15, 6), (3, 5, 6)):
        r = normal(3, *shape).cuda().requires_grad_()
        y = layers.linear(x, w, None, "tanh", r)
        gy = normal(4, *y.shape).cuda()
        for graph in (False, True):
            gx, gw, gr = torch.autograd.grad(y, (x, w, r), gy, retain_graph=True, create_graph=graph)
            assert y.shape == (3, 5, 6) and gr.shape == r.shape and torch.equal(gr.reshape(15, 6), gy.reshape(15, 6))
            assert gx.shape == x.shape and gw.shape == w.shape
    sync()


def test_negated_views(layers):
    """The imaginary part of a conjugate is a view that torch negates when it is read."""
    c = torch.complex(normal(1, 40, 1), normal(2, 40, 1)).cuda()
    x, w = torch.conj(c).imag, torch.ones(4, 1, device="cuda")
    assert x.is_neg()
    want = layers.linear_forward(x.clone(), w, save=False)
    assert torch.equal(layers.linear_forward(x, w, save=False), want) and float(want.norm()) > 0
    b = torch.conj(torch.complex(normal(3, 1), normal(4, 1)).cuda()).imag
    got = layers.linear_forward(x.clone(), w[:1], b, save=False)
    assert b.is_neg() and torch.equal(got, layers.linear_forward(x.clone(), w[:1], b.clone(), save=False))
    sync()


class Elsewhere(torch.Tensor):
    """A tensor that says it is on another device, without memory there."""

    @staticmethod
    def __new__(cls, size, dtype=F32):
        return torch.Tensor._make_wrapper_subclass(cls, size, dtype=dtype, device="cuda:1")

    @classmethod
    def __torch_dispatch__(cls, f, types, args=(), kwargs=None):
        raise RuntimeError("no operation here")


def test_tensors_of_another_device_are_refused(layers):
    x, w, b, n = (torch.ones(s, device="cuda") for s in ((4, 8), (6, 8), (6,), (8,)))
    gy, z = torch.ones(4, 6, device="cuda"), torch.ones(4, 6, device="cuda")
    stats = torch.ones(4, 2, device="cuda")
    E = Elsewhere
    for call in (lambda: layers.linear_forward(E((4, 8)), w, b),
                 lambda: layers.linear_forward(x, E((6, 8)), b),
                 lambda: layers.linear_forward(x, w, E((6,))),
                 lambda: layers.linear(x, w, E((6,))),
                 lambda: layers.linear_forward(x, w, b, residual=E((4, 6))),
                 lambda: layers.linear_backward(E((4, 6)), x, w, z, "tanh"),
                 lambda: layers.linear_backward(gy, x, w, E((4, 6)), "tanh"),
                 lambda: layers.gated_forward(x, w, w, E((6,)), b),
                 lambda: layers.gated_forward(x, w, w, b, E((6,))),
                 lambda: layers.gated_backward(gy, x, w, w, E((2, 4, 6))),
                 lambda: layers.layer_norm_forward(x, E((8,)), n),
                 lambda: layers.layer_norm_forward(x, n, E((8,))),
                 lambda: layers.layer_norm_backward(x, x, E((8,)), stats),
                 lambda: layers.layer_norm_backward(x, x, n, E((4, 2)))):
        with pytest.raises(ValueError):
            call()
    sync()


def child(code, **env):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env={**os.environ, **env}, capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    return json.loads(r.stdout.strip().splitlines()[-1])


EDGES = """
import ctypes, json, torch
from paper_2607_11985_gb300 import layers
x, w = torch.ones(64, 256, device="cuda", dtype=torch.bfloat16), torch.ones(128, 256, device="cuda", dtype=torch.bfloat16)
def step():
    n, s = layers.layer_norm_forward(x)
    y, z = layers.linear_forward(n, w, None, "tanh")
    return layers.linear_backward(y, n, w, z, "tanh")
step()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph(keep_graph=True)
with torch.cuda.graph(graph):
    out = step()
rt = None
for line in open("/proc/self/maps"):
    if "libcudart" in line:
        rt = ctypes.CDLL(line.split()[-1].strip())
        break
n = ctypes.c_size_t()
handle = ctypes.c_void_p(graph.raw_cuda_graph())
assert rt.cudaGraphGetEdges(handle, None, None, None, ctypes.byref(n)) == 0
a, b, data = (ctypes.c_void_p * n.value)(), (ctypes.c_void_p * n.value)(), ((ctypes.c_ubyte * 8) * n.value)()
assert rt.cudaGraphGetEdges(handle, a, b, data, ctypes.byref(n)) == 0
print(json.dumps([n.value, sum(e[2] == 1 for e in data)]))
"""


def test_plain_stream_order_on_request():
    """VQC_PDL=0: no kernel of the layer operators is let in before the one ahead of it ends.
    Counted in a captured graph: edges, and those of them that are programmatic."""
    edges, programmatic = child(EDGES, VQC_PDL="1")
    assert edges >= 3 and programmatic >= 1
    edges, programmatic = child(EDGES, VQC_PDL="0")
    assert edges >= 3 and programmatic == 0


LIMIT = """
import json, torch
from paper_2607_11985_gb300 import binding as B, layers
def ran_out():
    try:
        B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)
        return False
    except B.VQCError as e:
        assert B.STATUS[e.status] == "VQC_ERR_DEVICE_CHECK" and "timed out" in str(e), e
        return True
def matrix(rows, cols, dtype):
    return torch.ones(rows, cols, dtype=dtype, device="cuda")
seen = []
for dtype, rows, out, inp in ((torch.bfloat16, 4096, 4096, 65536), (torch.float16, 2048, 1024, 65536),
                              (torch.float32, 1024, 1024, 16384), (torch.bfloat16, 128, 64, 1 << 20)):
    x, w = matrix(rows, inp, dtype), matrix(out, inp, dtype)
    for call in (lambda: layers.linear_forward(x, w, save=False), lambda: layers.gated_forward(x, w, w, save=False),
                 lambda: layers.linear_backward(matrix(rows, out, dtype), x, w, None, "none")):
        call()
        seen.append(ran_out())
        # the device and the library go on: torch's kernels, and a product without such waits
        assert float(x[:, 0].float().sum()) == rows
        y = layers.linear_forward(x[:1, :64].contiguous(), w[:8, :64].contiguous(), save=False)
        assert float(y.float().sum()) == 8 * 64 and not ran_out()
print(json.dumps(seen))
"""


def test_waits_that_run_out_end_the_kernel_and_are_reported():
    """With a limit of one microsecond the roles of the tensor-core products give up in the
    middle of their work, with copies and products in flight: the kernel ends, the status
    says so, and the device can be used as before."""
    seen = child(LIMIT, VQC_WAIT_NS="1000")
    assert len(seen) == 12 and sum(seen[:3]) == 3, seen
    assert sum(child(LIMIT, VQC_WAIT_NS="4000000000")) == 0


REPORTED = """
import json, torch
from paper_2607_11985_gb300 import binding as B, layers
x, w = torch.ones(4096, 65536, dtype=torch.bfloat16, device="cuda"), torch.ones(4096, 65536, dtype=torch.bfloat16, device="cuda")
few = torch.ones(2, 64, dtype=torch.bfloat16, device="cuda").requires_grad_()
small = torch.ones(8, 64, dtype=torch.bfloat16, device="cuda")
y = layers.linear(few, small)
layers.linear_forward(x, w, save=False)
torch.cuda.synchronize()
def status(call):
    try:
        call()
        return "VQC_OK"
    except B.VQCError as e:
        return B.STATUS[e.status]
def backward():
    try:
        torch.autograd.grad(y, few, torch.ones_like(y), retain_graph=True)
        return "VQC_OK"
    except RuntimeError as e:
        return "timed out" if "timed out" in str(e) else str(e)
calls = [lambda: layers.linear_forward(few.detach(), small), lambda: layers.gated_forward(few.detach(), small, small),
         lambda: layers.linear(few, small), lambda: layers.linear_backward(y.detach(), few.detach(), small, None),
         lambda: B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)]
before, during = [status(c) for c in calls[:4]], backward()
told = [status(calls[4]) for _ in range(2)]
print(json.dumps([before, during, told, status(calls[0]), status(calls[2])]))
"""


def test_a_wait_that_ran_out_is_reported_by_later_calls():
    """Nobody needs to ask: calls after the one whose wait ran out raise, under autograd too,
    until vqc_sync_check has reported it, once."""
    before, during, told, one, two = child(REPORTED, VQC_WAIT_NS="1000")
    assert before == ["VQC_ERR_DEVICE_CHECK"] * 4 and during == "timed out"
    assert told == ["VQC_ERR_DEVICE_CHECK", "VQC_OK"] and one == two == "VQC_OK"


def test_float_parts_of_large_operands(layers):
    """Operands of 2^8 and more are cut, not rounded, into their parts: the products that are left
    out are then 2^-22 of a term each, two of them, of its sign.  With random signs the 2-norm
    of the error is that of float sums (2^-24 sqrt(n / 3)) and of the cuts in a chunk (16 * 2^-25)
    besides."""
    rows, inp, out = 1024, 2048, 1024
    for a, b in ((1e3, 1e3), (1e3, 1.0), (1e18, 1e18)):
        x, w = normal(1, rows, inp, scale=a).cuda(), normal(2, out, inp, scale=b).cuda()
        y = layers.linear_forward(x, w, save=False)
        sync()
        want = x.double() @ w.double().t()
        limit = 2 * 2.0 ** -22 + 2.0 ** -24 * math.sqrt(inp / 3) + 16 * 2.0 ** -25
        assert float((y.double() - want).norm() / want.norm()) <= limit


CAPTURED = """
import json, torch
from paper_2607_11985_gb300 import binding as B, layers
x, w = torch.randn(256, 512, device="cuda").bfloat16(), torch.randn(128, 512, device="cuda").bfloat16()
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    y, z = layers.linear_forward(x, w, None, "gelu")
    g = layers.linear_backward(y, x, w, z, "gelu")
for t in (y, z) + tuple(g):
    t.zero_()
graph.replay()
torch.cuda.synchronize()
u, v = layers.linear_forward(x, w, None, "gelu")
h = layers.linear_backward(u, x, w, v, "gelu")
B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)
print(json.dumps([torch.equal(a, b) for a, b in zip((y, z) + tuple(g), (u, v) + tuple(h))]))
"""


def test_first_products_of_a_process_inside_a_capture():
    assert child(CAPTURED) == [True] * 5
