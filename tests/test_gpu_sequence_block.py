"""The sequence block (norms, projections, rotated heads, attention, dropout, then the hybrid halves): whole
sequences, their gradients, and tokens one by one over a cache."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def cuda_ready():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)


def attention_half(block, h, lengths, kept):
    """The first half of the block in float64, elementary operations; kept: factor of the branch's elements."""
    p = {n: v.detach().double().requires_grad_() for n, v in block.named_parameters() if not n.startswith("rest.")}
    x = h.detach().double().requires_grad_()
    batch, tokens, _ = x.shape
    d = x - x.mean(-1, keepdim=True)
    a = d / torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5) * p["norm_weight"] + p["norm_bias"]
    at = torch.arange(tokens, device=x.device)

    def turned(y, w):
        y = y.unflatten(-1, (-1, block.dim))
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w
        angle = (at[:, None] * block.frequencies)[None, :, None]
        c, s, n = angle.cos(), angle.sin(), block.dim // 2
        return torch.cat([y[..., :n] * c - y[..., n:] * s, y[..., n:] * c + y[..., :n] * s], -1)
    q, k = turned(a @ p["w_q"].t(), p["weight_q"]), turned(a @ p["w_k"].t(), p["weight_k"])
    v = (a @ p["w_v"].t()).unflatten(-1, (-1, block.dim))
    per = block.heads // block.groups
    k, v = (t.repeat_interleave(per, 2) for t in (k, v))
    seen = (at <= at[:, None]) & ((at[:, None] - at < block.window) | (at < block.sinks))
    z = torch.einsum("bihd,bjhd->bhij", q, k) * block.dim ** -0.5
    o = torch.einsum("bhij,bjhd->bihd", torch.softmax(torch.where(seen, z, -math.inf), -1), v)
    o = torch.where(at[None, :, None, None] < lengths[:, None, None, None], o, 0.0)
    return x + o.flatten(-2) @ p["w_o"].t() * kept, p, x


@pytest.mark.parametrize("dtype,limit", [(torch.float32, 3e-5), (torch.bfloat16, 0.04), (torch.float16, 0.005)])
def test_block_and_gradients(dtype, limit):
    """Limits: as those of the hybrid block, with ten roundings in a row of the results in between."""
    from paper_2607_11985_gb300.hybrid import SequenceBlock
    from tests import sequence_reference as ref
    block = SequenceBlock(48, 4, 2, 24, 3, window=7, sinks=2, dropout=0.25, dtype=dtype, seed=5, hidden=64)
    g = torch.Generator().manual_seed(6)
    h = torch.randn(2, 21, 48, generator=g).to(dtype).cuda().requires_grad_()
    gy = torch.randn(2, 21, 48, generator=g).to(dtype).cuda()
    lengths = torch.tensor([21, 13], dtype=torch.int32, device="cuda")
    rest, block.rest = block.rest, torch.nn.Identity()       # the first half alone: the rest has its own test
    for step in range(2):                                     # drawn anew in every pass
        y = block(h, lengths)
        kept = ref.kept((2, 21, 48), 0.25, 5, step).cuda().double() / 0.75
        params = {n: v for n, v in block.named_parameters()}
        got = torch.autograd.grad(y, [h] + list(params.values()), gy)
        want, p, x = attention_half(block, h, lengths, kept)
        wanted = torch.autograd.grad(want, [x] + [p[n] for n in params], gy.double())
        for name, a, b in zip(["y", "h"] + list(params), [y] + list(got), [want] + list(wanted)):
            d = (a.detach().double() - b.detach()).norm() / b.detach().norm()
            assert float(d) <= limit, (step, name, float(d))
    block.rest = rest
    grads = torch.autograd.grad(block(h, lengths), [h] + list(block.parameters()), gy)
    assert all(bool(t.isfinite().all()) for t in grads)


@pytest.mark.parametrize("dtype,limit", [(torch.float32, 2e-5), (torch.bfloat16, 0.03), (torch.float16, 0.004)])
def test_tokens_over_a_cache(dtype, limit):
    """A prompt, then token by token: what the whole sequence gives at their places."""
    from paper_2607_11985_gb300.hybrid import SequenceBlock
    block = SequenceBlock(64, 4, 1, 32, 4, window=5, sinks=1, dropout=0.5, dtype=dtype, seed=2, hidden=96).eval()
    h = torch.randn(3, 19, 64, generator=torch.Generator().manual_seed(3)).to(dtype).cuda()
    with torch.no_grad():
        whole = block(h)
    cache, t, parts = block.cache(3, 20), 0, []
    for new in (6, 1, 1, 2) + (1,) * 9:
        lengths = torch.full((3,), t + new, dtype=torch.int32, device="cuda")
        parts.append(block.step(h[:, t:t + new], cache, lengths))
        t += new
    assert t == 19
    d = (torch.cat(parts, 1).double() - whole.double()).norm() / whole.double().norm()
    assert float(d) <= limit, float(d)


def test_training_runs():
    from paper_2607_11985_gb300.hybrid import train_sequence
    losses = train_sequence(width=64, qubits=4, batch=4, tokens=33, steps=6, say=lambda *_: None)
    assert len(losses) == 6 and all(math.isfinite(v) for v in losses)
