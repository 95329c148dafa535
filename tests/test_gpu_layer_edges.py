"""Layer operators at the edges: of their types' range and bits, of torch's views, tangents
and devices, and of the time that they may take.
"""

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

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


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("rows,inp,out", [(512, 1024, 4), (8, 1000, 600)])
def test_gradients_of_float_outputs_round_once(layers, dtype, rows, inp, out):
    """dz is grad_y itself here, a float32 matrix: the gradients are its products in float
    sums, rounded once, so that no bit of dz is missing."""
    x, w, gy = normal(1, rows, inp, dtype=dtype), normal(2, out, inp, dtype=dtype), normal(3, rows, out)
    gx, gw, _ = layers.linear_backward(gy.cuda(), x.cuda(), w.cuda(), None, "none")
    sync()
    once(gx, gy.double(), w.double(), dtype, "gx")
    once(gw, gy.double().t(), x.double(), dtype, "gw")
