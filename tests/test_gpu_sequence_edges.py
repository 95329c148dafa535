"""Operators of a sequence and their block at the edges: an epsilon of nothing, gradients that have nowhere to go, strides of
axes of one, prompts over a cache, blocks whose forward pass is made twice, stacked and converted blocks."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

from tests import sequence_reference as ref
from tests.layers_reference import check

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    torch.cuda.set_device(0)
    from paper_2607_11985_gb300 import layers
    return layers


@pytest.fixture(autouse=True)
def errors_are_reported(layers):
    yield
    from paper_2607_11985_gb300 import binding as B
    torch.cuda.synchronize()
    B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)


def normal(seed, *shape, dtype=F32):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def wide(t):
    return None if t is None else t.detach().double()


def cpu(pair):
    return tuple(t.cpu() for t in pair)


def turns(dim):
    return torch.tensor([10000.0 ** (-2 * i / dim) for i in range(dim // 2)], dtype=torch.float64, device="cuda")


# -------------------------------------------------------------- norms and rotation

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("eps", [0.0, 1e-50])         # (the second is none as a float)
@pytest.mark.parametrize("batch,tokens,count,groups,dim", [
    (1, 1, 1, 1, 64), (2, 3, 3, 1, 64), (1, 5, 4, 2, 128), (2, 400, 3, 1, 64), (3, 700, 5, 3, 16), (2, 9, 3, 1, 33)])
def test_norm_rotary_without_epsilon(layers, dtype, eps, batch, tokens, count, groups, dim):
    """Heads in odd numbers, alone, many and few tokens; packs of elements and single ones."""
    q, k, gq, gk = (normal(i, batch, tokens, n, dim, dtype=dtype) for i, n in ((1, count), (2, groups), (3, count), (4, groups)))
    wq, wk, freq = normal(5, dim, dtype=dtype), normal(6, dim, dtype=dtype), turns(dim - dim % 2)
    at = torch.arange(tokens).expand(batch, tokens)
    y = layers.norm_rotary_forward(q, k, wq, wk, freq, eps=eps)
    back = layers.norm_rotary_backward(gq, gk, q, k, wq, wk, freq, eps=eps)
    for i, (x, w, g) in enumerate(((q, wq, gq), (k, wk, gk))):
        want = ref.norm_rotary(wide(x).cpu(), wide(w).cpu(), freq.cpu(), at, eps, wide(g).cpu(), dtype)
        for name, got in (("y", y[i]), ("gx", back[i]), ("gw", back[2 + i])):
            check(got, want[name], dtype, 1, name + "qk"[i])


def test_frequencies_have_no_gradient(layers):
    """One that would be lost is refused, and a tangent."""
    import torch.autograd.forward_ad as fwd
    q, k, v, n = normal(1, 2, 3, 4, 8), normal(2, 2, 3, 2, 8), normal(3, 2, 3, 2, 8), torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    caches = torch.zeros(2, 2, 5, 2, 8, device="cuda")
    learned = turns(8).requires_grad_()
    for call in (lambda: layers.norm_rotary(q, k, None, None, learned), lambda: layers.norm_rotary(q.clone().requires_grad_(), k, None, None, learned),
                 lambda: layers.norm_rotary_step(q, k, v, *caches, n, None, None, learned)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    assert torch.equal(layers.norm_rotary(q, k, None, None, learned.detach())[0], layers.norm_rotary_forward(q, k, None, None, learned)[0])
    with fwd.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            layers.norm_rotary(q, k, None, None, fwd.make_dual(turns(8), turns(8)))


def test_step_refuses_caches_that_meet(layers):
    """Two views of one tensor are taken where no place of one is one of the other: decided as by listing the places.  What is
    written is what two tensors get (with the same strides and offsets: packs of elements are added in another order)."""
    batch, capacity, groups, dim = 2, 3, 2, 8
    q, k, v = normal(1, batch, 2, 4, dim), normal(2, batch, 2, groups, dim), normal(3, batch, 2, groups, dim)
    n, memory = torch.tensor([2, 3], dtype=torch.int32, device="cuda"), torch.zeros(1000, device="cuda")
    counts = [0, 0]
    for strides in ((48, 16, 8), (96, 32, 8), (96, 16, 48), (100, 33, 9), (96, 32, 16), (16, 100, 8), (200, 16, 8)):
        at = torch.as_strided(torch.arange(1000), (batch, capacity, groups, dim), (*strides, 1)).reshape(-1)
        for shift in (-131, -96, -48, -33, -32, -16, -9, -8, -7, -1, 0, 1, 7, 8, 9, 10, 16, 17, 24, 32, 40, 47, 48, 64, 72, 96, 100, 104, 131, 300):
            ck, cv = (memory.as_strided((batch, capacity, groups, dim), (*strides, 1), 300 + s) for s in (0, shift))
            meet = bool(torch.isin(at, at + shift).any())
            counts[meet] += 1
            memory.zero_()
            if meet:
                with pytest.raises(ValueError, match="cache_k and cache_v"):
                    layers.norm_rotary_step(q, k, v, ck, cv, n)
                assert not bool(memory.any())
            else:
                layers.norm_rotary_step(q, k, v, ck, cv, n)
                apart = [torch.zeros(1000, device="cuda").as_strided((batch, capacity, groups, dim), (*strides, 1), 300 + s) for s in (0, shift)]
                layers.norm_rotary_step(q, k, v, *apart, n)
                assert torch.equal(ck, apart[0]) and torch.equal(cv, apart[1])
    assert min(counts) > 20, counts
    # the capacity's last place left out of one and the first of the other; other strides
    buffer = torch.zeros(batch, 4, groups, dim, device="cuda")
    for ck, cv in ((buffer[:, :3], buffer[:, 1:]), (buffer[:, :3], buffer.view(batch, groups, 4, dim).transpose(1, 2)[:, :3])):
        with pytest.raises(ValueError, match="cache_k and cache_v"):
            layers.norm_rotary_step(q, k, v, ck, cv, n)
    assert not bool(buffer.any())


# -------------------------------------------------------------- attention

@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("batch,tokens,count,groups,dim", [(1, 200, 4, 2, 64), (2, 140, 1, 1, 128), (3, 1, 2, 1, 64), (1, 1, 1, 1, 128)])
def test_strides_of_axes_of_one_are_free(layers, dtype, batch, tokens, count, groups, dim):
    """As the header says of `aligned`, whose workspace is then enough."""
    from paper_2607_11985_gb300 import binding as B

    def odd(seed, heads):
        x = normal(seed, batch, tokens, heads, dim, dtype=dtype)
        strides = [s if n > 1 else 8 * s + 3 for n, s in zip(x.shape[:3], x.stride()[:3])]
        return x, torch.as_strided(x, x.shape, strides + [1])

    def heads(x):
        return ctypes.byref(B.vqc_heads(x.data_ptr(), *x.stride()[:3]))
    plain, odd_ones = zip(*(odd(i, n) for i, n in ((1, count), (2, groups), (3, groups), (4, count))))
    (q, k, v, g), (q1, k1, v1, g1) = plain, odd_ones
    code, stream = {BF16: B.VQC_BF16, F16: B.VQC_F16}[dtype], torch.cuda.current_stream().cuda_stream
    sizes = (batch, tokens, count, groups, dim)
    o, saved = layers.attention_forward(q, k, v, 50, 2)
    grads = layers.attention_backward(g, q, k, v, o, saved, 50, 2)
    for mode in (0, 1):
        need = B.vqc_attention_workspace_bytes(mode, code, *sizes, 50, 2, 1)
        space = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        if mode == 0:
            assert need == 0
            out, lse = torch.empty_like(o), torch.empty_like(saved)
            B.vqc_attention_forward(code, *sizes, heads(q1), heads(k1), heads(v1), 50, 2, dim ** -0.5, None, out.data_ptr(), lse.data_ptr(), None, 0, stream)
            assert torch.equal(out, o) and torch.equal(lse, saved)
        else:
            got = [torch.empty_like(t) for t in grads]
            B.vqc_attention_backward(code, *sizes, heads(g1), heads(q1), heads(k1), heads(v1), o.data_ptr(), saved.data_ptr(), 50, 2, dim ** -0.5, None,
                                     *(t.data_ptr() for t in got), space.data_ptr(), need, stream)
            assert all(torch.equal(a, b) for a, b in zip(got, grads))
    o1, saved1 = layers.attention_forward(q1, k1, v1, 50, 2)
    assert torch.equal(o1, o) and torch.equal(saved1, saved)
    assert all(torch.equal(a, b) for a, b in zip(layers.attention_backward(g1, q1, k1, v1, o1, saved1, 50, 2), grads))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("batch,tokens,count,groups,dim,window,sinks,lengths", [
    (1, 9000, 8, 8, 64, 64, 1500, None), (1, 9000, 8, 8, 64, 300, 1500, [8800]), (3, 4400, 8, 8, 64, 100, 2176, [4400, 4000, 1]), (2, 7000, 4, 2, 128, 40, 3000, None)])
def test_attention_with_many_first_tokens(layers, dtype, batch, tokens, count, groups, dim, window, sinks, lengths):
    """So many that their queries are cut into fewer pieces than windows, or not at all."""
    q, k, v, g = (normal(i, batch, tokens, n, dim, dtype=dtype) for i, n in ((1, count), (2, groups), (3, groups), (4, count)))
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want = ref.attention(*(wide(t) for t in (q, k, v, g)), window, sinks, None, lengths, dtype)
    o, saved = layers.attention_forward(q, k, v, window, sinks, lengths=n)
    check(o, cpu(want["o"]), dtype, 1.5, "o")
    grads = layers.attention_backward(g, q, k, v, o, saved, window, sinks, lengths=n)
    for name, x in zip(("gq", "gk", "gv"), grads):
        check(x, cpu(want[name]), dtype, 2, name)
    for a, b in zip(layers.attention_backward(g, q, k, v, o, saved, window, sinks, lengths=n), grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,count,groups,dim,capacity,window,sinks,lengths", [
    (2, 300, 4, 1, 64, 700, None, 0, [300, 555]), (1, 129, 6, 2, 128, 400, 60, 3, [390]), (2, 65, 2, 2, 80, 65, 17, 1, [65, 40]),
    (1, 200, 4, 2, 33, 200, None, 0, [200]), (1, 70, 2, 1, 192, 1500, 1000, 2, [1400])])
def test_prompt_over_a_cache(layers, dtype, batch, tokens, count, groups, dim, capacity, window, sinks, lengths):
    """Many new tokens at once, into an empty and a filled cache; the first of them at no position."""
    q, ck, cv = normal(1, batch, tokens, count, dim, dtype=dtype), normal(2, batch, capacity, groups, dim, dtype=dtype), normal(3, batch, capacity, groups, dim, dtype=dtype)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want = ref.attention_step(wide(q), wide(ck), wide(cv), lengths, window, sinks, None, dtype)
    for b, m in enumerate(lengths):
        ck[b, m:], cv[b, m:] = math.nan, math.inf
    check(layers.attention_step(q, ck, cv, n, window, sinks), cpu(want), dtype, 1.5, "o")


@pytest.mark.parametrize("dim", [64, 128])
def test_captured_float16_backward(layers, dim):
    """Its norms are set to zero between the kernels: captured, and replayed on new inputs."""
    q, k, v, g = (normal(i, 2, 200, n, dim, dtype=F16) for i, n in ((1, 4), (2, 2), (3, 2), (4, 4)))

    def step():
        o, saved = layers.attention_forward(q, k, v, 70, 1)
        return (o, *layers.attention_backward(g, q, k, v, o, saved, 70, 1))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for scale in (1.0, 2.0 ** -8, 2.0 ** 4):
        g.copy_(normal(9, 2, 200, 4, dim) * scale)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, step()):
            assert torch.equal(a, b)


# -------------------------------------------------------------- the block

def blocks(count, dtype=F32, **given):
    """Blocks whose hybrid half has a test of its own; what they drop is y == h."""
    from paper_2607_11985_gb300.hybrid import SequenceBlock
    made = [SequenceBlock(48, 4, 2, 24, 3, window=7, sinks=2, dropout=0.5, dtype=dtype, hidden=64, **given) for _ in range(count)]
    for b in made:
        b.rest = torch.nn.Identity()
    return torch.nn.Sequential(*made)


def gradients(model, call, h, gy):
    model.zero_grad()
    x = h.detach().requires_grad_()
    y = call(x)
    y.backward(gy)
    return [y.detach(), x.grad] + [p.grad.clone() for p in model.parameters()]


@pytest.mark.parametrize("reentrant", [False, True])
def test_checkpointed_block(layers, reentrant):
    """A forward pass that is made again for its backward draws what it has drawn: gradients are those of the plain block."""
    from torch.utils.checkpoint import checkpoint
    model, h, gy = blocks(2), normal(1, 2, 21, 48), normal(2, 2, 21, 48)
    for seed in (1, 2):
        torch.manual_seed(seed)
        want = gradients(model, model, h, gy)
        torch.manual_seed(seed)
        got = gradients(model, lambda x: checkpoint(model, x, use_reentrant=reentrant), h, gy)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("reentrant", [False, True])
def test_checkpointed_block_that_counts_its_passes(layers, reentrant):
    """Draws that are counted in the block would be others in the second pass: refused there, and given by the caller."""
    from torch.utils.checkpoint import checkpoint
    block, h, gy = blocks(1, seed=5)[0], normal(1, 2, 21, 48), normal(2, 2, 21, 48)
    with pytest.raises(RuntimeError, match="draws"):
        gradients(block, lambda x: checkpoint(block, x, use_reentrant=reentrant), h, gy)
    state, other = torch.tensor([5, 40], device="cuda"), torch.tensor([5, 41], device="cuda")
    count = block.draws.clone()
    want = gradients(block, lambda x: block(x, None, state), h, gy)
    got = gradients(block, lambda x: checkpoint(block, x, None, state, use_reentrant=reentrant), h, gy)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(block.draws, count)
    kept = ref.kept(h.shape, 0.5, 5, 40).cuda()
    assert torch.equal(want[0] == h, ~kept)
    assert not torch.equal(block(h, None, other) == h, ~kept)


def test_stacked_blocks_draw_apart(layers):
    """Blocks without a seed draw from torch's generator: each its own, anew in every pass, again from the same seed."""
    model, h = blocks(3), normal(1, 4, 40, 48)

    def masks():
        with torch.no_grad():
            return [block(h) == h for block in model]
    torch.manual_seed(3)
    first, second = masks(), masks()
    drawn = first + second
    for i, a in enumerate(drawn):
        assert abs(float(a.double().mean()) - 0.5) < 5 * 0.5 / math.sqrt(a.numel())
        for b in drawn[:i]:          # independent draws agree in half of the places
            assert abs(float((a == b).double().mean()) - 0.5) < 5 * 0.5 / math.sqrt(a.numel())
    torch.manual_seed(3)
    assert all(torch.equal(a, b) for a, b in zip(masks(), first))


def test_captured_block_draws_anew(layers):
    """Torch's generator goes on in the replays; a replay's backward draws what its forward has drawn."""
    block, h, gy = blocks(1)[0], normal(1, 2, 21, 48), normal(2, 2, 21, 48)

    def step():
        x = h.detach().requires_grad_()
        y = block(x)
        branch, = torch.autograd.grad(y, block.w_o, gy)
        return y.detach(), branch
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, branch = step()
    seen = []
    with torch.no_grad():
        q, k, v = block._heads(h)
        q, k = layers.norm_rotary(q, k, block.weight_q, block.weight_k, block.frequencies)
        a = layers.attention(q, k, v, block.window, block.sinks).flatten(-2).reshape(-1, 96).double()
    for _ in range(3):
        graph.replay()
        kept = (y != h)
        seen.append(kept.clone())
        want = torch.where(kept, 2 * gy, 0.0).reshape(-1, 48).double().t() @ a
        assert float((branch.double() - want).norm() / want.norm()) < 1e-5        # sums of 42 terms of another mask: 1
    assert not torch.equal(seen[0], seen[1]) and not torch.equal(seen[1], seen[2])


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_converted_block(layers, dtype):
    """What has a type of its own in a block (the frequencies; the circuit's angles and the projection behind it) keeps it."""
    from paper_2607_11985_gb300.hybrid import SequenceBlock
    made = {"window": 7, "sinks": 2, "seed": 5, "hidden": 64}
    block, other = SequenceBlock(48, 4, 2, 24, 3, **made).to(dtype), SequenceBlock(48, 4, 2, 24, 3, dtype=dtype, **made)
    assert block.frequencies.dtype == torch.float64
    for a, b in zip(block.state_dict().values(), other.state_dict().values()):
        assert a.dtype == b.dtype and torch.equal(a, b)
    h, gy = normal(1, 2, 21, 48, dtype=dtype), normal(2, 2, 21, 48, dtype=dtype)
    assert torch.equal(block(h), other(h))
    block(h).backward(gy)
    again = block.to(F32)           # gradients go with their parameters
    for p in again.parameters():
        assert p.dtype == F32 and p.grad.dtype == F32
    assert torch.equal(again.frequencies, other.frequencies) and bool(again(h.float()).isfinite().all())
