"""The operators of a sequence on the GPU against their definitions in 64 bits (sequence_reference):
types, head layouts, lengths from none to several tiles, windows that end inside tiles, strides, empty rows,
values that are not finite in places that nothing sees, streams and captured calls."""
import json
import math
import os
import subprocess
import sys

import pytest
import torch

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
def errors_are_reported():
    yield
    from paper_2607_11985_gb300 import binding as B
    torch.cuda.synchronize()
    B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)


def normal(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def heads(seed, batch, tokens, count, dim, dtype, stride=0, scale=1.0):
    """[batch, tokens, count, dim], a slice of rows that are `stride` elements longer"""
    wide = normal(seed, batch, tokens, count * dim + stride, dtype=dtype, scale=scale)
    return wide[..., :count * dim].unflatten(-1, (count, dim))


def child(code, **env):
    r = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                       env={**os.environ, **env}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    return json.loads(r.stdout.strip().splitlines()[-1])


def wide(t):
    return None if t is None else t.detach().double()


def cpu(pair):
    return tuple(t.cpu() for t in pair)


# -------------------------------------------------------------- dropout

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,stride,residual,p", [
    (1, 1, 0, True, 0.5), (3, 7, 0, False, 0.3), (5, 8, 8, True, 0.1), (33, 12, 4, True, 0.1), (64, 256, 0, True, 0.1),
    (7, 1001, 3, True, 0.9), (2, 40000, 0, False, 0.25), (129, 96, 32, False, 0.0)])
def test_dropout(layers, dtype, rows, cols, stride, residual, p):
    x = normal(1, rows, cols + stride, dtype=dtype)[:, :cols]
    res = normal(2, rows, cols + 2 * stride, dtype=dtype)[:, :cols] if residual else None
    gy = normal(3, rows, cols, dtype=dtype)
    seed, offset = 0xFEDCBA9876543210, 2 ** 40 + 5
    want = ref.dropout(wide(x).cpu(), None if res is None else wide(res).cpu(), wide(gy).cpu(), p, seed, offset, dtype)
    y = layers.dropout_forward(x, p, seed, offset, res)
    check(y, want["y"], dtype, 1, "y")
    gx = layers.dropout_backward(gy, p, seed, offset)
    check(gx, want["gx"], dtype, 1, "gx")
    assert torch.equal(gx == 0, (~ref.kept((rows, cols), p, seed, offset)).cuda() | (gy == 0))
    # the same through autograd, with a seed in device memory
    state = torch.tensor([seed - 2 ** 64, 2 ** 40], device="cuda")
    leaves = [t.detach().requires_grad_() for t in ([x, res] if residual else [x])]
    out = layers.dropout(leaves[0], p, state, 5, leaves[1] if residual else None)
    assert torch.equal(out, y)
    grads = torch.autograd.grad(out, leaves, gy)
    assert torch.equal(grads[0], gx) and (not residual or torch.equal(grads[1], gy))


def test_dropped_elements_count_as_zero(layers):
    """Also infinities and NaN; and the fraction that is kept."""
    x, res = torch.full((64, 512), math.nan, device="cuda"), normal(1, 64, 512)
    on = ref.kept((64, 512), 0.25, 7, 0).cuda()
    y = layers.dropout_forward(x, 0.25, 7, 0, res)
    assert torch.equal(y[~on], res[~on]) and bool(y[on].isnan().all())
    assert abs(float(on.double().mean()) - 0.75) < 5 * math.sqrt(0.25 * 0.75 / on.numel())
    other = layers.dropout_forward(torch.ones_like(res), 0.25, 7, 1) != 0
    assert 0.5 < float((other == on).double().mean()) < 0.75           # 0.625 where draws are independent


def test_captured_dropout_draws_anew(layers):
    x, gy = normal(1, 32, 64), normal(2, 32, 64)
    state = torch.tensor([11, 0], device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layers.dropout_forward(x, 0.5, state)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        leaf = x.detach().requires_grad_()
        y = layers.dropout(leaf, 0.5, state, 3)
        gx, = torch.autograd.grad(y, leaf, gy)
        state[1] += 1
    for step in range(3):
        graph.replay()
        on = ref.kept((32, 64), 0.5, 11, 3 + step).cuda()
        assert torch.equal(y.detach(), torch.where(on, 2 * x, 0.0)) and torch.equal(gx, torch.where(on, 2 * gy, 0.0))


# -------------------------------------------------------------- norms and rotation

def turns(dim, base=10000.0):
    return torch.tensor([base ** (-2 * i / dim) for i in range(dim // 2)], dtype=torch.float64, device="cuda")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,count,groups,dim,turned,stride,weights,far", [
    (1, 1, 1, 1, 64, 64, 0, True, 0), (2, 3, 4, 2, 128, 128, 0, True, 1000), (3, 33, 5, 1, 80, 48, 24, True, 10 ** 6),
    (2, 17, 3, 3, 33, 32, 5, True, 100), (1, 9, 2, 1, 256, 256, 8, True, 2 ** 30), (2, 5, 2, 2, 1, 0, 0, True, 0),
    (1, 300, 8, 2, 64, 32, 0, False, 77), (2, 40, 2, 1, 16, 16, 4, False, 5), (4, 1, 3, 1, 24, 6, 0, True, 9),
    (2, 700, 12, 4, 40, 40, 0, True, 31)])
def test_norm_rotary(layers, dtype, batch, tokens, count, groups, dim, turned, stride, weights, far):
    q, k = heads(1, batch, tokens, count, dim, dtype, stride), heads(2, batch, tokens, groups, dim, dtype, stride)
    gq, gk = heads(3, batch, tokens, count, dim, dtype, stride), heads(4, batch, tokens, groups, dim, dtype)
    wq, wk = (normal(5 + i, dim, dtype=dtype) if weights else None for i in range(2))
    freq = turns(turned) if turned else None
    pos = (far + torch.arange(batch * tokens, device="cuda", dtype=torch.int32).reshape(batch, tokens)) if far else None
    at = pos if far else torch.arange(tokens, device="cuda").expand(batch, tokens)
    yq, yk = layers.norm_rotary_forward(q, k, wq, wk, freq, pos)
    back = layers.norm_rotary_backward(gq, gk, q, k, wq, wk, freq, pos)
    for name, x, w, g, y, gx, gw in (("q", q, wq, gq, yq, back[0], back[2]), ("k", k, wk, gk, yk, back[1], back[3])):
        want = ref.norm_rotary(wide(x).cpu(), None if w is None else wide(w).cpu(), None if freq is None else freq.cpu(), at.cpu(), 1e-6, wide(g).cpu(), dtype)
        check(y, want["y"], dtype, 1, "y" + name)
        check(gx, want["gx"], dtype, 1, "gx" + name)
        assert (gw is None) == (w is None)
        if w is not None:
            check(gw, want["gw"], dtype, 1, "gw" + name)
    if weights:
        leaves = [t.detach().requires_grad_() for t in (q, k, wq, wk)]
        y = layers.norm_rotary(*leaves, freq, pos)
        assert torch.equal(y[0], yq) and torch.equal(y[1], yk)
        for a, b in zip(torch.autograd.grad(y, leaves, (gq, gk)), back):
            assert torch.equal(a, b)
        one, = torch.autograd.grad(layers.norm_rotary(*leaves, freq, pos)[1], leaves[1:2], gk)
        assert torch.equal(one, back[1])
    if pos is not None and batch == 1:
        assert torch.equal(layers.norm_rotary_forward(q, k, wq, wk, freq, pos[0])[0], yq)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,count,groups,dim", [(5, 1, 4, 2, 64), (3, 3, 2, 1, 33), (2, 2, 8, 8, 128)])
def test_norm_rotary_step_writes_its_places_only(layers, dtype, batch, tokens, count, groups, dim):
    capacity, freq = 20, turns(dim - dim % 2)
    q, k, v = heads(1, batch, tokens, count, dim, dtype, 3), heads(2, batch, tokens, groups, dim, dtype, 3), heads(3, batch, tokens, groups, dim, dtype)
    ck, cv = heads(4, batch, capacity, groups, dim, dtype, 8), heads(5, batch, capacity, groups, dim, dtype).transpose(1, 2).contiguous().transpose(1, 2)
    wq, wk = normal(6, dim, dtype=dtype), normal(7, dim, dtype=dtype)
    lengths = torch.tensor([tokens, capacity, capacity + 1, 0, 7][:batch], dtype=torch.int32, device="cuda")
    old_k, old_v = ck.clone(), cv.clone()
    version = ck._version
    y = layers.norm_rotary_step(q, k, v, ck, cv, lengths, wq, wk, freq)
    assert ck._version > version
    pos = (lengths[:, None] - tokens + torch.arange(tokens, device="cuda")).int()
    want_q, want_k = layers.norm_rotary_forward(q, k, wq, wk, freq, pos)
    assert torch.equal(y, want_q)
    for b in range(batch):
        for t in range(tokens):
            at = int(pos[b, t])
            if 0 <= at < capacity:
                old_k[b, at], old_v[b, at] = want_k[b, t], v[b, t]
    assert torch.equal(ck, old_k) and torch.equal(cv, old_v)


# -------------------------------------------------------------- attention

CASES = [
    # batch, tokens, heads, groups, dim, window, sinks, lengths, stride
    (1, 1, 1, 1, 64, None, 0, None, 0),
    (2, 2, 2, 1, 16, None, 0, None, 0),
    (1, 127, 2, 2, 128, None, 0, None, 0),
    (2, 128, 4, 1, 64, None, 0, None, 8),
    (1, 129, 3, 3, 72, 5, 0, None, 0),
    (3, 200, 6, 2, 80, 64, 3, [200, 131, 0], 16),
    (4, 65, 2, 1, 33, 1, 2, [65, 1, 0, 64], 5),
    (1, 300, 2, 1, 128, 130, 1, None, 5),
    (2, 257, 4, 4, 40, 100, 300, [257, 129], 0),
    (1, 640, 2, 1, 64, 128, 4, None, 0),
    (1, 700, 8, 2, 96, None, 0, [650], 0),
    (1, 70, 2, 1, 160, None, 0, None, 0),
    (2, 100, 2, 2, 256, 33, 2, [100, 50], 8),
    (1, 1100, 1, 1, 128, 256, 130, None, 0),
    (1, 5000, 2, 1, 64, 64, 130, [4900], 0),      # keys that stay visible: several pieces of far queries
    (1, 4500, 2, 2, 128, 300, 2, None, 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,count,groups,dim,window,sinks,lengths,stride", CASES)
def test_attention(layers, dtype, batch, tokens, count, groups, dim, window, sinks, lengths, stride):
    q, k, v = (heads(i, batch, tokens, n, dim, dtype, stride) for i, n in ((1, count), (2, groups), (3, groups)))
    g = heads(4, batch, tokens, count, dim, dtype, stride)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    sight = {"window": window, "sinks": sinks, "lengths": n}
    want = ref.attention(*(wide(t) for t in (q, k, v, g)), window, sinks, None, lengths, dtype)
    o, saved = layers.attention_forward(q, k, v, **sight)
    check(o, cpu(want["o"]), dtype, 1.5, "o")
    lse = want["lse"].cpu()
    got = saved.double().cpu()
    assert torch.equal(got.isinf(), lse.isinf())
    assert float((got - lse).nan_to_num(0, 0, 0).abs().max()) <= 2e-5
    assert torch.equal(layers.attention_forward(q, k, v, save=False, **sight), o)
    grads = layers.attention_backward(g, q, k, v, o, saved, **sight)
    for name, x in zip(("gq", "gk", "gv"), grads):
        check(x, cpu(want[name]), dtype, 2, name)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    y = layers.attention(*leaves, **sight)
    assert torch.equal(y, o)
    for a, b in zip(torch.autograd.grad(y, leaves, g), grads):
        assert torch.equal(a, b)
    only_q, none, none_too = layers.attention_backward(g, q, k, v, o, saved, **sight, need_kv=False)
    assert torch.equal(only_q, grads[0]) and none is None and none_too is None
    assert torch.equal(torch.autograd.grad(layers.attention(q, k, leaves[2], **sight), leaves[2], g)[0], grads[2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 20])
def test_tokens_behind_a_sequence_are_not_read(layers, dtype, dim):
    """NaN in the padding reaches no output and no gradient."""
    lengths = torch.tensor([150, 3, 0], dtype=torch.int32, device="cuda")
    t = {}
    for i, (name, count) in enumerate((("q", 4), ("k", 2), ("v", 2), ("g", 4))):
        t[name] = heads(i, 3, 200, count, dim, dtype)
    filled = {name: x.clone() for name, x in t.items()}
    for x in filled.values():
        for b, n in enumerate(lengths.tolist()):
            x[b, n:] = math.nan
    for sight in ({"window": 40, "sinks": 2}, {}):
        results = []
        for x in (t, filled):
            o, saved = layers.attention_forward(x["q"], x["k"], x["v"], lengths=lengths, **sight)
            results.append((o, saved, *layers.attention_backward(x["g"], x["q"], x["k"], x["v"], o, saved, lengths=lengths, **sight)))
        for a, b in zip(*results):
            assert torch.equal(a, b) and not bool(a.isnan().any())
        o, _, gq, gk, gv = results[0]
        for x in (o, gq, gk, gv):
            for b, n in enumerate(lengths.tolist()):
                assert not bool(x[b, n:].any())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_large_and_small_scores(layers, dtype):
    """Scores up to thousands: one key takes a row; maxima that grow along the keys."""
    q, k, v, g = (heads(i, 1, 384, 2, 64, dtype) for i in range(4))
    q, k = q * 8, (k * torch.linspace(0.1, 8, 384, device="cuda")[None, :, None, None]).to(dtype)
    want = ref.attention(*(wide(t) for t in (q, k, v, g)), None, 0, None, None, dtype)
    o, saved = layers.attention_forward(q, k, v)
    check(o, cpu(want["o"]), dtype, 2, "o")
    for name, x in zip(("gq", "gk", "gv"), layers.attention_backward(g, q, k, v, o, saved)):
        check(x, cpu(want[name]), dtype, 4, name)


@pytest.mark.parametrize("scale", [2.0 ** -12, 2.0 ** -3, 2.0 ** 6])
def test_float16_gradients_of_any_size(layers, scale):
    """p and ds are small where many keys share a row: their products keep the type's precision."""
    q, k, v = (heads(i, 1, 600, 2, 64, F16, scale=0.5) for i in range(3))
    g = heads(3, 1, 600, 2, 64, F16, scale=scale)
    want = ref.attention(*(wide(t) for t in (q, k, v, g)), None, 0, None, None, F16)
    o, saved = layers.attention_forward(q, k, v)
    for name, x in zip(("gq", "gk", "gv"), layers.attention_backward(g, q, k, v, o, saved)):
        # Results below 2^-14 are multiples of 2^-24: rounding is off by up to 2^-25 each, whatever their size, so
        # that the 2-norm of the error is two roundings of the result's and at most sqrt(count) 2^-25.
        value = want[name][0]
        fixed = math.sqrt(value.numel()) * 2.0 ** -25 / float(value.norm()) * 2 ** 11
        check(x, cpu(want[name]), F16, 2 + fixed, name)


def test_gradients_against_differences(layers):
    """In float32 with a window, sinks and padding, through norm, rotation and attention."""
    n = torch.tensor([23, 9], dtype=torch.int32, device="cuda")
    q, k, v = heads(1, 2, 23, 4, 16, F32), heads(2, 2, 23, 2, 16, F32), heads(3, 2, 23, 2, 16, F32)
    w, freq = 1 + 0.2 * normal(4, 16), turns(16)
    g = heads(5, 2, 23, 4, 16, F32)

    def loss(q, k, v, w):
        a, b = layers.norm_rotary(q, k, w, None, freq)
        return (layers.attention(a, b, v, 6, 2, 0.7, n) * g).sum(dtype=torch.float64)
    leaves = [t.detach().requires_grad_() for t in (q, k, v, w)]
    grads = torch.autograd.grad(loss(*leaves), leaves)
    for i, (x, gx) in enumerate(zip((q, k, v, w), grads)):
        step = normal(10 + i, *x.shape)
        args = [q, k, v, w]
        values = []
        for sign in (1, -1):
            args[i] = x + sign * 1e-2 * step
            values.append(loss(*args))
        slope = float(values[0] - values[1]) / 2e-2
        size = float(gx.norm() * step.norm())
        # second-order central differences: 1e-4 of third derivatives, and float outputs over the step
        assert abs(slope - float((gx.double() * step).sum())) <= 3e-3 * size, (i, slope)


# -------------------------------------------------------------- over a cache

STEPS = [
    # batch, tokens, heads, groups, dim, capacity, window, sinks, lengths
    (1, 1, 1, 1, 64, 1, None, 0, [1]),
    (3, 1, 8, 2, 128, 700, None, 0, [700, 64, 1]),
    (4, 1, 4, 4, 64, 300, 100, 4, [300, 101, 0, 99]),
    (2, 3, 6, 2, 80, 333, 17, 3, [333, 2]),
    (2, 2, 16, 1, 33, 150, None, 0, [149, 75]),
    (1, 5, 16, 2, 128, 2100, 1500, 1, [2099]),
    (2, 1, 4, 1, 256, 200, 64, 2, [200, 130]),
    (1, 1, 2, 2, 16, 5000, None, 0, [4999]),
    (1, 9, 8, 1, 64, 130, 5, 130, [130]),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch,tokens,count,groups,dim,capacity,window,sinks,lengths", STEPS)
def test_attention_step(layers, dtype, batch, tokens, count, groups, dim, capacity, window, sinks, lengths):
    q = heads(1, batch, tokens, count, dim, dtype, 3)
    ck, cv = heads(2, batch, capacity, groups, dim, dtype, 8), heads(3, batch, capacity, groups, dim, dtype)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    want = ref.attention_step(wide(q), wide(ck), wide(cv), lengths, window, sinks, None, dtype)
    for b, m in enumerate(lengths):       # places from the length on are not read
        ck[b, m:], cv[b, m:] = math.nan, math.inf
    o = layers.attention_step(q, ck, cv, n, window, sinks)
    check(o, cpu(want), dtype, 1.5, "o")
    assert torch.equal(layers.attention_step(q, ck, cv, n, window, sinks), o)
    over = n + (n == capacity).int() * 5                 # lengths beyond the capacity count as it
    assert torch.equal(layers.attention_step(q, ck, cv, over, window, sinks), o)
    # another order of memory: heads before places
    turned = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (ck, cv)]
    assert torch.equal(layers.attention_step(q, *turned, n, window, sinks), o)


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_one_by_one_as_a_whole_sequence(layers, dtype):
    """norm_rotary_step and attention_step over a growing cache, against norm_rotary and attention."""
    batch, tokens, count, groups, dim, window, sinks = 2, 37, 4, 2, 64, 9, 2
    q, k, v = heads(1, batch, tokens, count, dim, dtype), heads(2, batch, tokens, groups, dim, dtype), heads(3, batch, tokens, groups, dim, dtype)
    wq, wk, freq = normal(4, dim, dtype=dtype), normal(5, dim, dtype=dtype), turns(dim)
    a, b = layers.norm_rotary(q, k, wq, wk, freq)
    whole = layers.attention(a, b, v, window, sinks)
    ck, cv = torch.full((batch, 40, groups, dim), math.nan, dtype=dtype, device="cuda"), torch.full((batch, 40, groups, dim), math.nan, dtype=dtype, device="cuda")
    want = ref.attention(wide(a), wide(b), wide(v), None, window, sinks, None, None, dtype)["o"]
    t = 0
    for new in (5, 1, 1, 3) + (1,) * 27:
        n = torch.full((batch,), t + new, dtype=torch.int32, device="cuda")
        s = slice(t, t + new)
        x = layers.norm_rotary_step(q[:, s], k[:, s], v[:, s], ck, cv, n, wq, wk, freq)
        assert torch.equal(x, a[:, s]) and torch.equal(ck[:, s], b[:, s])
        o = layers.attention_step(x, ck, cv, n, window, sinks)
        check(o, tuple(z[:, s].cpu() for z in want), dtype, 1.5, "o at %d" % t)
        t += new
    check(whole, cpu(want), dtype, 1.5, "whole")


def test_step_refuses_shared_places(layers):
    """A cache is written: its places have to lie apart; views of one tensor for both caches are fine."""
    q, k, n = heads(2, 2, 1, 4, 8, F32), heads(3, 2, 1, 2, 8, F32), torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    ck, cv = torch.zeros(2, 5, 2, 8, device="cuda"), torch.zeros(2, 5, 2, 8, device="cuda")
    over = torch.zeros(200, device="cuda")
    bad = [
        lambda: layers.norm_rotary_step(q, k, k, ck, ck, n), lambda: layers.norm_rotary_step(q, ck[:, 2:3], k, ck, cv, n),
        lambda: layers.norm_rotary_step(q, k, cv[:, 2:3], ck, cv, n),
        lambda: layers.norm_rotary_step(q, k, k, over.as_strided((2, 5, 2, 8), (64, 8, 8, 1)), cv, n),
        lambda: layers.norm_rotary_step(q, k, k, over.as_strided((2, 5, 2, 8), (80, 16, 7, 1)), cv, n),
        lambda: layers.norm_rotary_step(q.clone().requires_grad_(), k, k, ck, cv, n),
        lambda: layers.norm_rotary_step(q, k, k, ck, cv, n, torch.ones(8, device="cuda", requires_grad=True)),
        lambda: layers.attention_step(q.clone().requires_grad_(), ck, cv, n),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)
    assert not bool(ck.any()) and not bool(cv.any())
    # keys beside values in one tensor; heads before places
    both, turned = torch.zeros(2, 5, 2, 2, 8, device="cuda"), torch.zeros(2, 2, 2, 5, 8, device="cuda")
    with torch.no_grad():
        layers.norm_rotary_step(q.clone().requires_grad_(), k, k, ck, cv, n)
    layers.norm_rotary_step(q, k, k, both[:, :, 0], both[:, :, 1], n)
    layers.norm_rotary_step(q, k, k, turned[0].transpose(1, 2), turned[1].transpose(1, 2), n)
    for a, b in ((both[:, :, 0], ck), (both[:, :, 1], cv), (turned[0].transpose(1, 2), ck), (turned[1].transpose(1, 2), cv)):
        assert torch.equal(a, b)


# -------------------------------------------------------------- streams, graphs, repeats

@pytest.mark.parametrize("dtype", [F32, BF16])
def test_captured_step_on_another_stream(layers, dtype):
    """A whole training step of the operators captured, replayed on new inputs; two graphs share nothing."""
    q, k, v, g = (heads(i, 2, 150, 2, 64, dtype) for i in range(4))
    w, freq = normal(9, 64, dtype=dtype), turns(64)
    state = torch.tensor([5, 0], device="cuda")

    def step(q, k, v, g):
        leaves = [t.detach().requires_grad_() for t in (q, k, v, w)]
        a, b = layers.norm_rotary(*leaves[:2], leaves[3], leaves[3], freq)
        y = layers.dropout(layers.attention(a, b, leaves[2], 50, 1), 0.1, state, residual=leaves[0])
        return (y.detach(), *torch.autograd.grad(y, leaves, g))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        eager = step(q, k, v, g)
    torch.cuda.current_stream().wait_stream(stream)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        inputs = [t.clone() for t in (q, k, v, g)]
        with torch.cuda.graph(graph):
            out = step(*inputs)
        graphs.append((graph, inputs, out))
    for a in graphs[0][1]:
        a.mul_(0.5)
    for graph, _, _ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(graphs[1][2], eager):
        assert torch.equal(a, b)
    for a, b in zip(graphs[0][2], step(*graphs[0][1])):
        assert torch.equal(a, b)


def test_results_repeat(layers):
    q, k, v, g = (heads(i, 2, 900, 8 if i in (0, 3) else 2, 128, BF16) for i in range(4))
    first = None
    for _ in range(4):
        o, saved = layers.attention_forward(q, k, v, 300, 4)
        now = (o, saved, *layers.attention_backward(g, q, k, v, o, saved, 300, 4))
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))


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
seen = []
for dtype, dim, window in ((torch.bfloat16, 128, None), (torch.float16, 64, 700), (torch.bfloat16, 40, None)):
    q, k, v = (torch.ones(2, 4096, n, dim, dtype=dtype, device="cuda") for n in (8, 2, 2))
    o, saved = torch.ones_like(q), torch.zeros(2, 8, 4096, device="cuda")
    for call in (lambda: layers.attention_forward(q, k, v, window, 3), lambda: layers.attention_backward(q, q, k, v, o, saved, window, 3)):
        for _ in range(4):
            call()
            seen.append(ran_out())
            # the device and the library go on
            assert float(q[:, 0].float().sum()) == 2 * 8 * dim
            w = layers.attention_step(q[:, :1], k, v, torch.full((2,), 9, dtype=torch.int32, device="cuda"))
            assert bool((w == 1).all()) and not ran_out()
print(json.dumps(seen))
"""


def test_waits_that_run_out_end_the_kernel_and_are_reported(layers):
    """With a limit of one microsecond the roles of the tensor-core kernels give up with copies and products in
    flight: the kernel ends, the status says so, and the device can be used as before."""
    seen = child(LIMIT, VQC_WAIT_NS="1000")
    assert len(seen) == 24 and any(seen[:4]) and any(seen[4:8]), seen
    assert not any(child(LIMIT, VQC_WAIT_NS="4000000000"))


# -------------------------------------------------------------- refusals

def test_refusals(layers):
    x, q, k = normal(1, 4, 8), heads(2, 2, 3, 4, 8, F32), heads(3, 2, 3, 2, 8, F32)
    n, freq = torch.tensor([3, 3], dtype=torch.int32, device="cuda"), turns(8)
    ck = torch.zeros(2, 5, 2, 8, device="cuda")
    bad = [
        lambda: layers.dropout(x, 1.0, 1), lambda: layers.dropout(x, -0.1, 1), lambda: layers.dropout(x, math.nan, 1),
        lambda: layers.dropout(x, 0.1, torch.tensor([1, 2], dtype=torch.int32, device="cuda")), lambda: layers.dropout(x, 0.1, torch.tensor([1, 2])),
        lambda: layers.dropout(x, 0.1, 1, 0, x[:, :4]), lambda: layers.dropout(x, 0.1, 1, 0, x.half()), lambda: layers.dropout(x.cpu(), 0.1, 1),
        lambda: layers.norm_rotary(q, k[:, :2]), lambda: layers.norm_rotary(q, k.half()), lambda: layers.norm_rotary(q[0], k[0]),
        lambda: layers.norm_rotary(q, k, x[0, :7]), lambda: layers.norm_rotary(q, k, None, None, freq.float()),
        lambda: layers.norm_rotary(q, k, None, None, turns(10)), lambda: layers.norm_rotary(q, k, None, None, freq, n.long()),
        lambda: layers.norm_rotary(q, k, None, None, freq, n), lambda: layers.norm_rotary(q, k, eps=-1.0),
        lambda: layers.norm_rotary(heads(1, 1, 1, 1, 264, F32), heads(1, 1, 1, 1, 264, F32)), lambda: layers.rotary_frequencies(7),
        lambda: layers.norm_rotary_step(q, k, k, ck, ck[:, :4], n), lambda: layers.norm_rotary_step(q, k, k, ck, ck.half(), n),
        lambda: layers.norm_rotary_step(q, k, k, ck[:, :1].expand(2, 5, 2, 8), ck, n), lambda: layers.norm_rotary_step(q, k, k, ck, ck, None),
        lambda: layers.norm_rotary_step(q, k, k, ck.clone().requires_grad_(), ck, n), lambda: layers.norm_rotary_step(q, k, k, ck, ck, n.long()),
        lambda: layers.attention(q, k, k, 0), lambda: layers.attention(q, k, k, -3), lambda: layers.attention(q, k, k, 4, -1),
        lambda: layers.attention(q, k, k, scale=0.0), lambda: layers.attention(q, k, k, scale=math.inf), lambda: layers.attention(q, k, k, scale=math.nan),
        lambda: layers.attention(q[:, :, :3], k, k), lambda: layers.attention(q, k, k[..., :4]), lambda: layers.attention(q, k, k[:, :2]),
        lambda: layers.attention(q, k, k, lengths=n[:1]), lambda: layers.attention(q, k, k, lengths=n.long()),
        lambda: layers.attention(q, k, k, lengths=n.cpu()), lambda: layers.attention(q.double(), k.double(), k.double()),
        lambda: layers.attention_backward(q, q, k, k, q, torch.zeros(2, 3, 4, device="cuda")),
        lambda: layers.attention_backward(q[:, :2], q, k, k, q, torch.zeros(2, 4, 3, device="cuda")),
        lambda: layers.attention_step(q, ck, ck[:, :4], n), lambda: layers.attention_step(q, ck, ck, None), lambda: layers.attention_step(q, ck[:1], ck[:1], n),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % i)
    # tangents are refused, and second derivatives
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level():
        with pytest.raises(RuntimeError, match="forward-mode"):
            layers.attention(fwd.make_dual(q, q), k, k)
    leaf = q.clone().requires_grad_()
    for y in (layers.dropout(leaf, 0.5, 1), layers.norm_rotary(leaf, k)[0], layers.attention(leaf, k, k)):
        first, = torch.autograd.grad(y.square().sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="once only"):
            torch.autograd.grad(first.sum(), leaf)
    # nothing to do
    none = q[:0]
    assert layers.attention(none, k[:0], k[:0]).shape == none.shape and layers.norm_rotary(none, k[:0])[0].shape == none.shape
    assert layers.attention_step(q[:, :0], ck, ck, n).shape == (2, 0, 4, 8) and layers.dropout(x[:0], 0.5, 1).shape == (0, 8)
    gw = layers.norm_rotary_backward(none, k[:0], none, k[:0], x[0], x[1])[2:]
    assert all(not bool(t.any()) for t in gw)
