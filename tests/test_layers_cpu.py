"""Classical operators without a GPU: argument checks of the C entry points and of
the Python calls, workspace sizes, and the 64-bit reference that the GPU tests use
(its gradients against torch's float64 autograd)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2607_11985_gb300 import binding as B  # noqa: E402
from tests import layers_reference as ref  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_11985_gb300 import build
    build.build()


A = 1 << 20    # an address that is never read: every call below is refused


def linear(dtype=1, out_dtype=1, rows=4, inp=8, out=6, x=A, ldx=8, w=A, ldw=8, b=None, act=2, res=None, ldr=0, y=A,
           saved=None):
    return B.lib().vqc_linear_forward(dtype, out_dtype, rows, inp, out, x, ldx, w, ldw, b, act, res, ldr, y, saved,
                                      None, 0, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(dtype=-1), dict(out_dtype=2), dict(rows=-1), dict(rows=1 << 31), dict(inp=0), dict(out=0),
    dict(out=1 << 31), dict(ldx=7), dict(ldw=7), dict(res=A, ldr=5), dict(x=None), dict(w=None), dict(y=None),
    dict(act=6), dict(act=-1), dict(x=A + 1), dict(w=A + 1), dict(b=A + 1), dict(y=A + 8), dict(saved=A + 4)])
def test_linear_refusals(bad):
    assert linear(**bad) == 1
    assert "vqc_linear_forward" in B.vqc_last_error()


def test_backward_refusals():
    L = B.lib()

    def lin(dtype=1, gy=A, ldg=6, x=A, w=A, saved=A, gx=A, gw=A, gb=A, ws=A, nbytes=1 << 30, act=2):
        return L.vqc_linear_backward(dtype, dtype, 4, 8, 6, gy, ldg, x, 8, w, 8, saved, act, gx, gw, gb, ws, nbytes,
                                     None)
    assert lin(gy=None) == 1 and lin(saved=None) == 1 and lin(x=None) == 1 and lin(w=None) == 1 and lin(ldg=5) == 1
    assert lin(gx=A + 8) == 1 and lin(ws=A + 16) == 1 and lin(dtype=9) == 1
    assert lin(ws=None) == 8 and lin(nbytes=16) == 8

    def gat(gwu=A, gbu=A, saved=A, wu=A, nbytes=1 << 30):
        return L.vqc_gated_backward(1, 4, 8, 6, A, 6, A, 8, A, wu, 8, saved, 3, A, A, gwu, A, gbu, A, nbytes, None)
    assert gat(gwu=None) == 1 and gat(gbu=None) == 1 and gat(saved=None) == 1 and gat(wu=None) == 1
    assert gat(nbytes=0) == 8
    assert L.vqc_gated_forward(1, 4, 8, 6, A, 8, A, None, 8, None, None, 3, A, None, None, 0, None) == 1

    def norm(dtype=0, rows=4, cols=8, x=A, ld=8, eps=1e-5, y=A):
        return L.vqc_layer_norm_forward(dtype, rows, cols, x, ld, None, None, eps, y, None, None)
    assert norm(dtype=3) == 1 and norm(rows=-1) == 1 and norm(cols=0) == 1 and norm(ld=7) == 1 and norm(x=None) == 1
    assert norm(eps=-1.0) == 1 and norm(eps=float("nan")) == 1 and norm(y=A + 4) == 1 and norm(x=A + 2) == 1

    def back(gy=A, stats=A, gw=A, ws=A, nbytes=1 << 30):
        return L.vqc_layer_norm_backward(0, 4, 8, gy, 8, A, 8, None, stats, A, gw, None, ws, nbytes, None)
    assert back(gy=None) == 1 and back(stats=None) == 1 and back(ws=None) == 8 and back(nbytes=8) == 8


def test_calls_without_rows_launch_nothing():
    assert linear(rows=0, x=None, y=None) == 0
    L = B.lib()
    assert L.vqc_layer_norm_forward(0, 0, 8, None, 8, None, None, 1e-5, None, None, None) == 0
    assert L.vqc_layer_norm_backward(0, 0, 8, None, 8, None, 8, None, None, None, None, None, None, 0, None) == 0


def test_workspace_sizes():
    L = B.lib()
    for mode in (0, 1):
        for rows in (0, 1, 7, 64, 1000, 8192):
            for inp, out in ((1, 1), (16, 12), (1024, 12), (517, 1031), (2048, 2048)):
                n = L.vqc_linear_workspace_bytes(mode, 1, 1, rows, inp, out, inp, inp, out, 2, 1)
                m = L.vqc_gated_workspace_bytes(mode, 1, rows, inp, out, inp, inp, 1)
                assert n % 256 == 0 and m % 256 == 0
                # never more than the operands, a copy of each and 256 MB of cut sums
                assert max(n, m) <= 64 * (rows + 64) * (inp + 8 + out + 8) + 16 * inp * out + (1 << 28)
    big = 2 ** 64 - 1
    assert L.vqc_linear_workspace_bytes(2, 1, 1, 4, 8, 6, 8, 8, 6, 0, 1) == big
    assert L.vqc_linear_workspace_bytes(0, 1, 2, 4, 8, 6, 8, 8, 6, 0, 1) == big
    assert L.vqc_linear_workspace_bytes(0, 1, 1, 4, 8, 6, 7, 8, 6, 0, 1) == big
    assert L.vqc_gated_workspace_bytes(0, 7, 4, 8, 6, 8, 8, 1) == big
    assert L.vqc_layer_norm_workspace_bytes(-1, 8) == big and L.vqc_layer_norm_workspace_bytes(5, 0) == big


def test_python_refuses_host_tensors():
    from paper_2607_11985_gb300 import layers
    x, w = torch.ones(4, 8), torch.ones(6, 8)
    for call in (lambda: layers.linear(x, w), lambda: layers.gated(x, w, w), lambda: layers.layer_norm(x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


@pytest.mark.parametrize("name", ["none", "relu", "gelu", "silu", "tanh", "sigmoid"])
def test_reference_gradients(name):
    f = {"none": lambda z: z, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
         "tanh": torch.tanh, "sigmoid": torch.sigmoid}[name]
    g = torch.Generator().manual_seed(1)
    x, w, u, b, c, gy = (torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True)
                         for s in ((5, 7), (4, 7), (4, 7), (4,), (4,), (5, 4)))
    one = ref.linear(x, w, b, name, None, gy, torch.float32, torch.float32)
    want = torch.autograd.grad(f(x @ w.t() + b), (x, w, b), gy.detach())
    for key, v in zip(("gx", "gw", "gb"), want):
        assert float((one[key][0] - v).abs().max()) <= 1e-12
    two = ref.gated(x, w, u, b, c, name, gy, torch.float32)
    want = torch.autograd.grad(f(x @ w.t() + b) * (x @ u.t() + c), (x, w, u, b, c), gy.detach())
    for key, v in zip(("gx", "gw", "gup", "gb", "gbup"), want):
        assert float((two[key][0] - v).abs().max()) <= 1e-12


def test_reference_norm_gradients():
    g = torch.Generator().manual_seed(2)
    x, w, b, gy = (torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True)
                   for s in ((5, 9), (9,), (9,), (5, 9)))
    one = ref.layer_norm(x, w, b, 1e-5, gy, torch.float32)
    y = torch.nn.functional.layer_norm(x, (9,), w, b, 1e-5)
    assert float((one["y"][0] - y).abs().max()) <= 1e-12
    for key, v in zip(("gx", "gw", "gb"), torch.autograd.grad(y, (x, w, b), gy.detach())):
        assert float((one[key][0] - v).abs().max()) <= 1e-12
