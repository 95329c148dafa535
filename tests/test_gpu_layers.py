"""Layer norm, linear and gated on the GPU against the definitions in 64 bits.

The bounds are derived in tests/layers_reference.py.  Covered: the three types
and the mixed ones, every activation, one row to many, odd sizes, sizes inside
and across tiles, strides, misaligned addresses and other layouts, rows with
infinities and NaN, no rows, products cut along the contraction, offsets past 32
bits, other streams, graph capture, repeatability, autograd, and gradients
against differences.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from tests import layers_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
ACTS = ["none", "relu", "gelu", "silu", "tanh", "sigmoid"]


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


def strided(t, how):
    """The same values on the GPU in another place and layout."""
    if t is None or how == "dense":
        return None if t is None else t.cuda()
    if how == "wide":        # rows of a wider tensor, 16-byte aligned rows where the type allows
        wide = torch.full((t.shape[0], t.shape[1] + 24), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 8:8 + t.shape[1]] = t.cuda()
        return wide[:, 8:8 + t.shape[1]]
    if how == "odd":         # an odd stride and a misaligned first element
        wide = torch.full((t.shape[0], t.shape[1] + 3), float("nan"), dtype=t.dtype, device="cuda")
        wide[:, 1:1 + t.shape[1]] = t.cuda()
        return wide[:, 1:1 + t.shape[1]]
    assert how == "columns"
    return t.t().contiguous().cuda().t()


def d64(t):
    return None if t is None else t.double()


SIZES = [(1, 1, 1), (1, 16, 12), (2, 512, 40), (3, 5, 7), (4, 1024, 260), (8, 264, 96), (9, 64, 200), (33, 1031, 17),
         (64, 64, 64), (65, 130, 33), (127, 257, 129), (128, 64, 256), (129, 520, 264), (300, 72, 1000),
         (1000, 16, 40), (517, 12, 1024), (257, 2048, 8), (256, 1024, 512), (1536, 320, 392)]


def run_linear(layers, rows, inp, out, dtype, act, residual, bias=True, out_dtype=None, how="dense", seed=1):
    out_dtype = out_dtype or dtype
    x, w = normal(seed, rows, inp, dtype=dtype), normal(seed + 1, out, inp, scale=inp ** -0.5, dtype=dtype)
    b = normal(seed + 2, out, scale=0.3, dtype=dtype) if bias else None
    res = normal(seed + 3, rows, out, dtype=out_dtype) if residual else None
    gy = normal(seed + 4, rows, out, dtype=out_dtype)
    want = ref.linear(d64(x), d64(w), d64(b), act, d64(res), d64(gy), dtype, out_dtype)
    X, W, R, G = (strided(t, how) for t in (x, w, res, gy))
    Bv = None if b is None else b.cuda()
    y, saved = layers.linear_forward(X, W, Bv, act, R, out_dtype)
    y2 = layers.linear_forward(X, W, Bv, act, R, out_dtype, save=False)
    gx, gw, gb = layers.linear_backward(G, X, W, saved, act, need_bias=bias)
    sync()
    assert y.dtype is out_dtype and gx.dtype is dtype and gw.dtype is dtype
    ref.check(y, want["y"], out_dtype, 1, "y")
    ref.check(y2, want["y"], out_dtype, 1, "y without saving")
    if saved is not None:
        ref.check(saved, want["z"], F32, 8, "z")
    ref.check(gx, want["gx"], dtype, 2, "gx")
    ref.check(gw, want["gw"], dtype, 2, "gw")
    if bias:
        ref.check(gb, want["gb"], dtype, 2, "gb")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k,size", list(enumerate(SIZES)))
def test_linear_sizes(layers, dtype, k, size):
    run_linear(layers, *size, dtype, ACTS[k % 6], residual=k % 2 == 0, bias=k % 3 != 1, seed=10 * k)


@pytest.mark.parametrize("dtype,out_dtype", [(BF16, BF16), (BF16, F32), (F16, F32), (F32, BF16), (F32, F16)])
@pytest.mark.parametrize("act", ACTS)
def test_linear_activations_and_types(layers, dtype, out_dtype, act):
    run_linear(layers, 70, 136, 50, dtype, act, residual=True, out_dtype=out_dtype, seed=300)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["wide", "odd", "columns"])
@pytest.mark.parametrize("size", [(3, 40, 24), (140, 96, 72), (133, 71, 45)])
def test_linear_layouts(layers, dtype, how, size):
    run_linear(layers, *size, dtype, "silu", residual=True, how=how, seed=400)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("size", [(4096, 64, 32), (24, 4096, 16), (5000, 48, 130), (20000, 8, 12)])
def test_linear_long_contractions(layers, dtype, size):
    """Products that are cut along the contraction: of the rows (gw), of the features."""
    run_linear(layers, *size, dtype, "tanh", residual=False, seed=500)


def run_gated(layers, rows, inp, out, dtype, act, bias=True, how="dense", seed=1):
    x = normal(seed, rows, inp, dtype=dtype)
    wg, wu = (normal(seed + i, out, inp, scale=inp ** -0.5, dtype=dtype) for i in (1, 2))
    bg, bu = (normal(seed + i, out, scale=0.3, dtype=dtype) if bias else None for i in (3, 4))
    gh = normal(seed + 5, rows, out, dtype=dtype)
    want = ref.gated(d64(x), d64(wg), d64(wu), d64(bg), d64(bu), act, d64(gh), dtype)
    X, WG, WU, G = (strided(t, how) for t in (x, wg, wu, gh))
    BG, BU = (None if b is None else b.cuda() for b in (bg, bu))
    h, saved = layers.gated_forward(X, WG, WU, BG, BU, act)
    h2 = layers.gated_forward(X, WG, WU, BG, BU, act, save=False)
    got = layers.gated_backward(G, X, WG, WU, saved, act, need_bias=bias)
    sync()
    ref.check(h, want["y"], dtype, 1, "h")
    ref.check(h2, want["y"], dtype, 1, "h without saving")
    for name, g in zip(("gx", "gw", "gup", "gb", "gbup"), got):
        if g is not None:
            ref.check(g, want[name], dtype, 2, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k,size", list(enumerate(SIZES)))
def test_gated_sizes(layers, dtype, k, size):
    run_gated(layers, *size, dtype, ACTS[(k + 2) % 6], bias=k % 3 != 1, seed=600 + 10 * k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["wide", "odd", "columns"])
def test_gated_layouts(layers, dtype, how):
    run_gated(layers, 133, 72, 104, dtype, "gelu", how=how, seed=900)


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_long_contraction(layers, dtype):
    run_gated(layers, 5000, 40, 24, dtype, "silu", seed=950)
    run_gated(layers, 20, 4100, 24, dtype, "silu", seed=960)


NORM_SIZES = [(1, 1), (5, 1), (1, 7), (64, 256), (33, 1000), (1021, 1001), (3, 4096), (130, 2048), (7, 8200), (2, 16384),
              (2, 40000), (3, 70001), (2000, 24)]


def run_norm(layers, rows, cols, dtype, how="dense", weight=True, bias=True, offset=0.0, eps=1e-5, seed=1):
    x = (normal(seed, rows, cols) * normal(seed + 1, rows, 1).exp() + offset).to(dtype)
    w = (1.0 + normal(seed + 2, cols, scale=0.3)).to(dtype) if weight else None
    b = normal(seed + 3, cols, scale=0.3, dtype=dtype) if bias else None
    gy = normal(seed + 4, rows, cols, dtype=dtype)
    want = ref.layer_norm(d64(x), d64(w), d64(b), eps, d64(gy), dtype)
    X, G = strided(x, how), strided(gy, how)
    W, Bv = (None if t is None else t.cuda() for t in (w, b))
    y, saved = layers.layer_norm_forward(X, W, Bv, eps)
    y2 = layers.layer_norm_forward(X, W, Bv, eps, save=False)
    gx, gw, gb = layers.layer_norm_backward(G, X, W, saved)
    sync()
    assert torch.equal(y, y2)
    for name, g in (("y", y), ("gx", gx), ("gw", gw), ("gb", gb)):
        value, bound = want[name]
        d = (g.double().cpu() - value).abs()
        assert bool((d <= bound).all()), (name, float((d / bound).max()))
    return y, gx, gw, gb, want


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k,size", list(enumerate(NORM_SIZES)))
def test_norm_sizes(layers, dtype, k, size):
    got = run_norm(layers, *size, dtype, weight=k % 4 != 2, bias=k % 3 != 1, seed=20 * k)
    if size[1] > 1:
        for name, g in zip(("y", "gx", "gw", "gb"), got):
            ref.check(g, got[4][name], dtype, 1, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("how", ["wide", "odd", "columns"])
@pytest.mark.parametrize("size", [(70, 96), (37, 333), (9, 9000)])
def test_norm_layouts(layers, dtype, how, size):
    run_norm(layers, *size, dtype, how=how, seed=700)


@pytest.mark.parametrize("size", [(40, 300), (5, 5000)])
def test_norm_large_mean_and_constant_rows(layers, size):
    run_norm(layers, *size, F32, offset=1000.0, seed=800)
    x = torch.full(size, 3.25, device="cuda")
    b = normal(1, size[1]).cuda()
    y, saved = layers.layer_norm_forward(x, None, b)
    gx, gw, gb = layers.layer_norm_backward(torch.ones_like(x), x, None, saved)
    sync()
    assert torch.equal(y, b.expand_as(y))          # no variance: the bias alone
    assert float(gx.abs().max()) <= 316.3 * 2.0 ** -20   # rstd = 1/sqrt(eps), g - mean(g) = rounding
    assert torch.equal(gw, torch.zeros_like(gw)) and torch.equal(gb, torch.full_like(gb, size[0]))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_with_infinities_and_nan_stay_alone(layers, dtype):
    rows, inp, out = 150, 96, 72
    for value in (math.inf, -math.inf, math.nan, torch.finfo(dtype).min):
        x = normal(1, rows, inp, dtype=dtype)
        x[5, 3] = x[140, 95] = value
        w, b = normal(2, out, inp, scale=inp ** -0.5, dtype=dtype), normal(3, out, dtype=dtype)
        clean = torch.ones(rows, dtype=torch.bool)
        clean[[5, 140]] = False
        X, W, Bv = x.cuda(), w.cuda(), b.cuda()
        y = layers.linear_forward(X, W, Bv, "none", save=False)
        h = layers.gated_forward(X, W, W, Bv, Bv, "relu", save=False)
        n = layers.layer_norm_forward(X, None, None, save=False)
        sync()
        want = ref.linear(d64(x[clean]), d64(w), d64(b), "none", None, None, dtype, dtype)["y"]
        ref.check(y.cpu()[clean], want, dtype, 1, "y")
        assert bool(torch.isfinite(h.cpu()[clean]).all() and torch.isfinite(n.cpu()[clean]).all())
        if not math.isfinite(value):
            assert not bool(torch.isfinite(y.cpu()[5]).any()) and not bool(torch.isfinite(y.cpu()[140]).any())
            expect = x[5].double() @ w.double().t() + b.double()
            assert torch.equal(torch.isnan(y.cpu()[5]), torch.isnan(expect))
            fine = ~torch.isnan(expect)
            assert torch.equal(y.cpu()[5].double()[fine], expect[fine])


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(layers, dtype):
    x, w, b = (torch.ones(s, dtype=dtype, device="cuda") for s in ((0, 24), (16, 24), (16,)))
    y, z = layers.linear_forward(x, w, b, "gelu")
    gx, gw, gb = layers.linear_backward(y, x, w, z, "gelu")
    h, zz = layers.gated_forward(x, w, w, b, b)
    got = layers.gated_backward(h, x, w, w, zz)
    n, stats = layers.layer_norm_forward(x, w[0])
    nx, nw, nb = layers.layer_norm_backward(n, x, w[0], stats)
    sync()
    assert y.shape == (0, 16) and h.shape == (0, 16) and n.shape == (0, 24) and gx.shape == nx.shape == (0, 24)
    for g in (gw, gb, got[1], got[2], got[3], got[4], nw, nb):
        assert bool((g == 0).all())


def test_offsets_past_32_bits(layers):
    rows, inp, out = 540_000, 16, 4096          # 2.2e9 outputs
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(rows, inp, generator=g, device="cuda").bfloat16()
    w = (torch.randn(out, inp, generator=g, device="cuda") / 4).bfloat16()
    y = layers.linear_forward(x, w, None, "none", save=False)
    n = layers.layer_norm_forward(y, None, None, save=False)
    gw = layers.linear_backward(y, x, w, None, need_x=False, need_bias=False)[1]
    sync()
    for part in (slice(0, 200), slice(524_200, 524_400), slice(rows - 200, rows)):
        want = x[part].cpu().double() @ w.cpu().double().t()
        assert float((y[part].cpu().double() - want).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
        yy = y[part].cpu().double()
        wn = (yy - yy.mean(1, keepdim=True)) / torch.sqrt(yy.var(1, unbiased=False, keepdim=True) + 1e-5)
        assert float((n[part].cpu().double() - wn).abs().max()) <= 2.0 ** -7 * float(wn.abs().max())
    want = torch.zeros(out, inp, dtype=torch.float64, device="cuda")
    for i in range(0, rows, 60_000):
        want += y[i:i + 60_000].double().t() @ x[i:i + 60_000].double()
    assert float((gw.double() - want).norm() / want.norm()) <= 2 * ref.U[BF16]
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_leading_axes_and_autograd(layers, dtype):
    x, res = (normal(i, 3, 50, 40, dtype=dtype).cuda() for i in (1, 2))
    w, wu = (normal(i, 24, 40, scale=0.2, dtype=dtype).cuda() for i in (3, 4))
    b, bu, nw, nb = (normal(i, n, dtype=dtype).cuda() for i, n in ((5, 24), (6, 24), (7, 40), (8, 40)))
    gy, gx0 = normal(9, 3, 50, 24, dtype=dtype).cuda(), normal(10, 3, 50, 40, dtype=dtype).cuda()
    leaf = lambda *ts: [t.clone().requires_grad_() for t in ts]   # noqa: E731

    a = leaf(x, w, b, normal(11, 3, 50, 24, dtype=dtype).cuda())
    y = layers.linear(a[0], a[1], a[2], "silu", a[3])
    got = torch.autograd.grad(y, a, gy)
    y1, z = layers.linear_forward(x, w, b, "silu", a[3].detach())
    want = layers.linear_backward(gy, x, w, z, "silu") + (gy,)
    assert torch.equal(y, y1) and all(torch.equal(p, q) for p, q in zip(got, want))

    a = leaf(x, w, wu, b, bu)
    h = layers.gated(*a, activation="tanh")
    got = torch.autograd.grad(h, a, gy)
    h1, z = layers.gated_forward(x, w, wu, b, bu, "tanh")
    assert torch.equal(h, h1)
    assert all(torch.equal(p, q) for p, q in zip(got, layers.gated_backward(gy, x, w, wu, z, "tanh")))

    a = leaf(x, nw, nb)
    n = layers.layer_norm(*a)
    got = torch.autograd.grad(n, a, gx0)
    n1, s = layers.layer_norm_forward(x, nw, nb)
    assert torch.equal(n, n1)
    assert all(torch.equal(p, q) for p, q in zip(got, layers.layer_norm_backward(gx0, x, nw, s)))

    # only some inputs need a gradient; an expanded gradient (a sum's)
    a = leaf(w)
    layers.linear(x, a[0], None, "none").sum().backward()
    ones = torch.ones(3, 50, 24, dtype=dtype, device="cuda")
    assert torch.equal(a[0].grad, layers.linear_backward(ones, x, w, None, need_x=False, need_bias=False)[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_repeatable_on_streams_and_in_graphs(layers, dtype):
    x, gy = normal(1, 700, 264, dtype=dtype).cuda(), normal(2, 700, 136, dtype=dtype).cuda()
    w, wu, b = normal(3, 136, 264, scale=0.1, dtype=dtype).cuda(), normal(4, 136, 264, dtype=dtype).cuda(), \
        normal(5, 136, dtype=dtype).cuda()
    nw = normal(6, 264, dtype=dtype).cuda()

    def step():
        n, s = layers.layer_norm_forward(x, nw)
        y, z = layers.linear_forward(n, w, b, "gelu")
        h, zz = layers.gated_forward(n, w, wu, b, b)
        out = [n, y, h] + list(layers.linear_backward(gy, n, w, z, "gelu")) + list(layers.gated_backward(gy, n, w, wu, zz))
        return out + list(layers.layer_norm_backward(out[3], x, nw, s))

    first = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x += 0                                     # produced on the other stream
        second = step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = step()
    for t in third:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, third))


def test_gradients_against_differences(layers):
    """Directional derivatives of L = sum gy * f by central differences of the
    float32 kernels (step 2^-7: the third derivatives leave about 1e-4, the float
    sums about 1e-4 of L's size)."""
    rows, inp, out, step = 40, 36, 28, 2.0 ** -7
    gy = normal(1, rows, out).cuda()
    res = normal(2, rows, out).cuda()
    cases = []
    for act in ("gelu", "silu", "tanh", "sigmoid", "none"):
        cases.append((lambda x, w, b, act=act: layers.linear(x, w, b, act, res),
                      [normal(3, rows, inp), normal(4, out, inp, scale=inp ** -0.5), normal(5, out)], gy))
        cases.append((lambda x, w, u, b, c, act=act: layers.gated(x, w, u, b, c, act),
                      [normal(6, rows, inp), normal(7, out, inp, scale=inp ** -0.5),
                       normal(8, out, inp, scale=inp ** -0.5), normal(9, out), normal(10, out)], gy))
    cases.append((lambda x, w, b: layers.layer_norm(x, w, b),
                  [normal(11, rows, inp), normal(12, inp), normal(13, inp)], normal(14, rows, inp).cuda()))
    for f, args, g in cases:
        args = [a.cuda() for a in args]
        leaves = [a.clone().requires_grad_() for a in args]
        grads = torch.autograd.grad(f(*leaves), leaves, g)
        for i in range(len(args)):
            v = normal(100 + i, *args[i].shape).cuda()
            v /= v.norm()
            loss = []
            for sign in (1, -1):
                moved = [a + sign * step * v if k == i else a for k, a in enumerate(args)]
                loss.append(float((f(*moved).double() * g.double()).sum()))
            diff = (loss[0] - loss[1]) / (2 * step)
            scale = float(grads[i].double().norm())
            assert abs(diff - float((grads[i].double() * v.double()).sum())) <= 2e-3 * scale, (i, diff)


def test_refusals_on_the_gpu(layers):
    x, w, b = torch.ones(4, 8, device="cuda"), torch.ones(6, 8, device="cuda"), torch.ones(6, device="cuda")
    for call in (lambda: layers.linear_forward(x, w[:, :7], b),
                 lambda: layers.linear_forward(x, w.half(), b),
                 lambda: layers.linear_forward(x, w, b[:5]),
                 lambda: layers.linear_forward(x, w, b, "softplus"),
                 lambda: layers.linear_forward(x, w, b, residual=torch.ones(4, 5, device="cuda")),
                 lambda: layers.linear_forward(x, w, b, residual=torch.ones(3, 6, device="cuda")),
                 lambda: layers.linear_forward(x, w, b, out_dtype=torch.float64),
                 lambda: layers.linear_forward(x.bfloat16(), w.bfloat16(), None, out_dtype=torch.float16),
                 lambda: layers.linear_forward(x.double(), w.double()),
                 lambda: layers.linear_backward(torch.ones(4, 6, device="cuda"), x, w, None, "gelu"),
                 lambda: layers.linear_backward(torch.ones(3, 6, device="cuda"), x, w, None),
                 lambda: layers.gated_forward(x, w, w[:5]),
                 lambda: layers.gated_backward(torch.ones(4, 6, device="cuda"), x, w, w, torch.ones(4, 6, device="cuda")),
                 lambda: layers.layer_norm_forward(x, b),
                 lambda: layers.layer_norm_backward(x, x, None, torch.ones(4, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    sync()


@pytest.mark.parametrize("which", ["layer_norm", "linear", "gated"])
def test_operands_left_out_and_second_derivatives(layers, which):
    """Every combination of optional operands and of inputs that need a gradient;
    create_graph gives the gradients and refuses theirs."""
    x, w, u = normal(1, 30, 16).cuda(), normal(2, 12, 16).cuda(), normal(3, 12, 16).cuda()
    b, c, r, nw, nb = (normal(i, *s).cuda() for i, s in ((4, (12,)), (5, (12,)), (6, (30, 12)), (7, (16,)), (8, (16,))))
    for given in range(4):
        first, second = given & 1, given >> 1
        if which == "layer_norm":
            ops, f = [x, nw if first else None, nb if second else None], layers.layer_norm
        elif which == "linear":
            ops, f = [x, w, b if first else None, r if second else None], \
                lambda x, w, b, r: layers.linear(x, w, b, "none" if given == 3 else "tanh", r)
        else:
            ops, f = [x, w, u, b if first else None, c if second else None], layers.gated
        present = [i for i, t in enumerate(ops) if t is not None]
        full = [t.clone().requires_grad_() if t is not None else None for t in ops]
        y = f(*full)
        gy = normal(9, *y.shape).cuda()
        want = dict(zip(present, torch.autograd.grad(y, [full[i] for i in present], gy, create_graph=True)))
        with pytest.raises(RuntimeError, match="once"):
            torch.autograd.grad(want[0].sum(), full[0])
        with torch.no_grad():
            assert torch.equal(f(*full), y) and not f(*full).requires_grad
        for i in present:                      # this input alone needs a gradient
            some = [t.clone().requires_grad_(k == i) if t is not None else None for k, t in enumerate(ops)]
            got, = torch.autograd.grad(f(*some), [some[i]], gy)
            assert torch.equal(got, want[i]), (given, i)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [2, 5, 8, 9, 13, 16, 17])
@pytest.mark.parametrize("inp,out", [(8, 3), (40, 30), (1000, 129), (4096, 64)])
def test_few_rows(layers, dtype, rows, inp, out):
    run_linear(layers, rows, inp, out, dtype, "gelu", residual=True, seed=1000 + rows)
    run_gated(layers, rows, inp, out, dtype, "silu", how="wide", seed=1100 + rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,inp,out", [(512, 4096, 12), (256, 4096, 256), (2048, 8192, 128)])
def test_float_outputs_of_deep_contractions(layers, dtype, rows, inp, out):
    """A float32 output keeps a float32 sum's accuracy at any depth.  With random signs
    the 2-norm of the error of a sum of n float32 roundings is about 2^-24 sqrt(n / 3)
    of the result's; sums of chunks of 256 that are cut (not rounded) at every 16 add
    16 * 2^-25.  Both together, and twice that for the spread: 2e-6 at n = 8192."""
    g = torch.Generator(device="cuda").manual_seed(rows + out)
    x = torch.randn(rows, inp, generator=g, device="cuda").to(dtype)
    w = (torch.randn(out, inp, generator=g, device="cuda") * inp ** -0.5).to(dtype)
    y = layers.linear_forward(x, w, None, "none", out_dtype=F32, save=False)
    h, z = layers.gated_forward(x, w, w, None, None, "none") if dtype == F32 else (None, None)
    sync()
    want = x.double() @ w.double().t()
    limit = 2 * (2.0 ** -24 * math.sqrt(inp / 3) + 16 * 2.0 ** -25)
    assert float((y.double() - want).norm() / want.norm()) <= limit
    if h is not None:
        assert float((h.double() - want * want).norm() / (want * want).norm()) <= 2 * limit


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_large_products_of_a_backward(layers, dtype):
    """Above 6e9 operations dz is one 16-bit matrix."""
    run_linear(layers, 2048, 1024, 1024, dtype, "gelu", residual=True, seed=1200)
    run_gated(layers, 1100, 1024, 1024, dtype, "silu", seed=1210)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(300, 200, 150), (77, 96, 640)])
def test_small_products_of_a_backward_round_once(layers, dtype, rows, inp, out):
    """Below, dz keeps twice the bits: what is left of its rounding (2^-16 or less of it)
    and of the float sums is far below the one rounding of a gradient, so that the
    gradients are as near as the rounded float64 ones (5 percent for what float sums move)."""
    x, w, u = normal(1, rows, inp, dtype=dtype), *(normal(i, out, inp, scale=inp ** -0.5, dtype=dtype) for i in (2, 3))
    gy = normal(4, rows, out, dtype=dtype)
    X, W, V, G = (t.cuda() for t in (x, w, u, gy))
    _, z = layers.linear_forward(X, W, None, "tanh")
    _, zz = layers.gated_forward(X, W, V)
    lin = layers.linear_backward(G, X, W, z, "tanh", need_bias=False)[:2]
    gat = layers.gated_backward(G, X, W, V, zz, need_bias=False)[:3]
    sync()
    a = ref.linear(d64(x), d64(w), None, "tanh", None, d64(gy), dtype, dtype)
    b = ref.gated(d64(x), d64(w), d64(u), None, None, "silu", d64(gy), dtype)
    for got, want in list(zip(lin, (a["gx"], a["gw"]))) + list(zip(gat, (b["gx"], b["gw"], b["gup"]))):
        exact = want[0]
        once = float((exact.to(dtype).double() - exact).norm())
        assert float((got.double().cpu() - exact).norm()) <= 1.05 * once


def test_float_parts_with_infinities_nan_and_large_values(layers):
    """Float products that run in bf16 parts keep float arithmetic's infinities, NaN and
    range: 3.4e38 would round to an infinite part."""
    rows, inp, out = 600, 1024, 520
    x, w, u = normal(1, rows, inp), normal(2, out, inp, scale=inp ** -0.5), normal(3, out, inp, scale=inp ** -0.5)
    x[5, 3], x[6, 4], x[7, 9], x[7, 10] = math.inf, math.nan, math.inf, -math.inf
    x[8, 11], w[:, 11] = 3.4e38, w[:, 11].clamp(-0.2, 0.2)
    X, W, V = x.cuda(), w.cuda(), u.cuda()
    y = layers.linear_forward(X, W, None, "none", save=False).cpu().double()
    h = layers.gated_forward(X, W, V, None, None, "sigmoid", save=False).cpu().double()
    sync()
    clean = torch.ones(rows, dtype=torch.bool)
    clean[5:9] = False
    want = x.double() @ w.double().t()
    ref.check(y[clean].float(), ref.linear(d64(x[clean]), d64(w), None, "none", None, None, F32, F32)["y"], F32, 8, "y")
    for row in (5, 6, 7):
        assert torch.equal(torch.isnan(y[row]), torch.isnan(want[row])), row
        fine = ~torch.isnan(want[row])
        assert torch.equal(y[row][fine], want[row][fine]), row
    assert bool(torch.isfinite(y[8]).all()) and float((y[8] - want[8]).norm() / want[8].norm()) <= 1e-6
    gate, up = torch.sigmoid(want), x.double() @ u.double().t()
    assert bool(torch.isfinite(h[clean]).all()) and bool(torch.isnan(h[6]).all())
    assert torch.equal(torch.isnan(h[5]), torch.isnan((gate * up)[5]))
    # gradients: an infinite incoming gradient reaches its row of gx and its column's row of gw, no more
    gy = normal(4, rows, out)
    gy[17, 33] = math.inf
    xc = normal(5, rows, inp)
    gx, gw, gb = layers.linear_backward(gy.cuda(), xc.cuda(), W, None, "none")
    sync()
    want_x, want_w = gy.double() @ w.double(), gy.double().t() @ xc.double()
    for got, exact in ((gx, want_x), (gw, want_w)):
        got = got.cpu().double()
        assert torch.equal(torch.isfinite(got), torch.isfinite(exact)) and torch.equal(torch.isnan(got), torch.isnan(exact))
        bad = ~torch.isfinite(exact)
        assert torch.equal(got[bad], exact[bad])
        assert float((got[~bad] - exact[~bad]).norm() / exact[~bad].norm()) <= 1e-6
    assert math.isinf(float(gb[33])) and bool(torch.isfinite(torch.cat([gb[:33], gb[34:]])).all())


def test_overflow_of_dz_stays_infinite(layers):
    """dg beyond float16's range is infinite in both forms of dz, and so are the gradients
    that it enters: not NaN."""
    rows, inp, out = 20, 48, 40
    x, wg, wu = normal(1, rows, inp, dtype=F16), normal(2, out, inp, dtype=F16), normal(3, out, inp, dtype=F16)
    gh = normal(4, rows, out, dtype=F16)
    X, WG, WU = x.cuda(), wg.cuda(), wu.cuda()
    _, z = layers.gated_forward(X, WG, WU, None, None, "none")
    j = int(z[1, 3].abs().cpu().argmax())
    gh[3, j] = 60000.0                             # times |u| > 2: beyond 65504
    assert float(z[1, 3, j].abs()) > 2
    gx, gw, gup, _, _ = layers.gated_backward(gh.cuda(), X, WG, WU, z, "none", need_bias=False)
    sync()
    # dg and du rounded to float16, infinite where they exceed it, and the products of these: an infinity, or
    # NaN where infinities of both signs meet
    z64, gh64 = z.cpu().double(), gh.double()
    dg, du = (gh64 * z64[1]).to(F16).double(), (gh64 * z64[0]).to(F16).double()
    assert bool(torch.isinf(dg[3, j]))
    for got, want in ((gx, dg @ wg.double() + du @ wu.double()), (gw, dg.t() @ x.double()), (gup, du.t() @ x.double())):
        got = got.cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        bad = torch.isinf(want)
        assert bool(bad.any()) and torch.equal(got[bad], want[bad])
        assert bool(torch.isfinite(got[torch.isfinite(want)]).all())
