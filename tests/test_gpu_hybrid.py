"""The hybrid block (layer norm, linear, circuit, gated feed-forward) against the same
block in float64: the oracle's expectations and adjoint gradients between
elementary torch operations."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import oracle as orc  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def cuda_ready():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


class OracleCircuit(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, spec):
        ctx.spec = spec
        ctx.save_for_backward(x, w)
        return torch.from_numpy(np.ascontiguousarray(orc.forward(spec, x.detach().numpy(), w.detach().numpy())))

    @staticmethod
    def backward(ctx, gE):
        x, w = (t.detach().numpy() for t in ctx.saved_tensors)
        dx, dw = orc.backward(ctx.spec, x, w, np.ascontiguousarray(gE.numpy()))
        return torch.from_numpy(dx), torch.from_numpy(dw), None


def reference(block, h):
    p = {k: v.detach().double().cpu().requires_grad_() for k, v in block.named_parameters()}
    x = h.detach().double().cpu().requires_grad_()

    def norm(v, w, b):
        d = v - v.mean(-1, keepdim=True)
        return d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5) * w + b
    a = torch.tanh(norm(x, p["norm1_weight"], p["norm1_bias"]) @ p["w_in"].t() + p["b_in"])
    z = OracleCircuit.apply(a.reshape(-1, a.shape[-1]), p["angles"], block.circuit.spec)
    y = x + z.reshape(x.shape[:-1] + (-1,)) @ p["w_out"].t() + p["b_out"]
    a = norm(y, p["norm2_weight"], p["norm2_bias"])
    g, u = a @ p["w_gate"].t(), a @ p["w_up"].t()
    return y + (g * torch.sigmoid(g) * u) @ p["w_down"].t(), p, x


@pytest.mark.parametrize("dtype,limit", [(torch.float32, 2e-5), (torch.bfloat16, 0.03), (torch.float16, 0.004)])
def test_block_and_gradients(dtype, limit):
    """Limits: in float32 the rounding of a few thousand terms, in the 16-bit types
    eight roundings in a row (2^-8 and 2^-11 each) of the results in between."""
    from paper_2607_11985_gb300.hybrid import HybridBlock
    block = HybridBlock(40, 5, depth=2, hidden=72, dtype=dtype, seed=3)
    g = torch.Generator().manual_seed(4)
    h = torch.randn(3, 11, 40, generator=g).to(dtype).cuda().requires_grad_()
    gy = torch.randn(3, 11, 40, generator=g).to(dtype).cuda()
    y = block(h)
    params = dict(block.named_parameters())
    got = torch.autograd.grad(y, [h] + list(params.values()), gy)
    want, p, x = reference(block, h)
    ref = torch.autograd.grad(want, [x] + [p[k] for k in params], gy.double().cpu())
    assert y.dtype is dtype and y.shape == h.shape
    for name, a, b in zip(["y", "h"] + list(params), [y] + list(got), [want] + list(ref)):
        d = (a.detach().double().cpu() - b.detach()).norm() / b.detach().norm()
        assert float(d) <= limit, (name, float(d))


def test_training_lowers_the_loss():
    from paper_2607_11985_gb300.hybrid import train
    losses = train(width=64, qubits=4, batch=256, steps=30, say=lambda *_: None)
    assert all(math.isfinite(v) for v in losses) and losses[-1] < 0.7 * losses[0], losses
