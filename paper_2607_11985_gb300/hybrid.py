"""A hybrid block: a circuit inside a residual network, and its training.

``HybridBlock`` is a residual block of two halves on features h [..., width]:

  h = h + W_out circuit(W_in norm(h))       a circuit in the place of a projection:
                                            features to n angles, <Z> of n qubits back
  h = h + W_down (act(norm(h) W_gate^T) * (norm(h) W_up^T))      a gated feed-forward

The features, norms and projections run in the features' type (float32, bfloat16 or
float16) in the ``layers`` kernels; the angles come out as float32 for the
complex64 circuit, and the float32 expectations go back into the residual
stream in the features' type: the last steps of the products on both sides of
the circuit.

``SequenceBlock`` stands before it where samples are tokens of sequences, [batch, tokens, width]:

  q, k, v = W_q norm(h), W_k norm(h), W_v norm(h)      in heads; keys and values in fewer
  q, k    = norms of each head, turned by their positions
  h       = h + dropout(W_o attention(q, k, v))         causal, through a window and over the first tokens

and then the two halves above.  In training a sequence goes through whole; ``step`` takes the next
tokens of sequences whose keys and values lie in a cache.

``python -m paper_2607_11985_gb300.hybrid`` trains one block on a synthetic task (``--tokens``: a
sequence block).
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B, layers, workloads as wl
from .circuit import Circuit


class _Block(torch.nn.Module):
    """A module some of whose tensors (``own_types``) have types of their own beside the features', which stay theirs where the
    module is converted to another one."""
    own_types = ()

    def _apply(self, fn, *args, **kwargs):
        own = [getattr(self, n) for n in self.own_types]
        own += [t.grad for t in own if t.grad is not None]
        kept = {id(t) for t in own}

        def moved(t):
            r = fn(t)
            return t.to(r.device) if id(t) in kept and r.dtype != t.dtype else r
        return super()._apply(moved, *args, **kwargs)


class HybridBlock(_Block):
    """See the module's text.  ``spec``: a circuit with one x angle per qubit
    (``workloads.CircuitSpec``), by default a layered ansatz of RY, RZ and CX."""
    own_types = ("angles", "w_out", "b_out")      # float32, as the circuit

    def __init__(self, width: int, qubits: int, depth: int = 2, hidden: int = 0, dtype=torch.float32, spec=None,
                 seed: int = 0):
        super().__init__()
        if spec is None:
            spec = wl.CircuitSpec(qubits, qubits, 2 * qubits * depth)
            for q in range(qubits):
                spec.add("RY", (q,), [("x", q)])
            for d in range(depth):
                for q in range(qubits):
                    spec.add("RY", (q,), [("w", 2 * (d * qubits + q))])
                    spec.add("RZ", (q,), [("w", 2 * (d * qubits + q) + 1)])
                for q in range(qubits if qubits > 1 else 0):
                    spec.add("CX", (q, (q + 1) % qubits))
        self.circuit = Circuit(spec, "c64")
        hidden = hidden or 4 * width
        g = torch.Generator().manual_seed(seed)

        def matrix(rows, cols, kind=dtype):
            return torch.nn.Parameter((torch.randn(rows, cols, generator=g) * cols ** -0.5).to(kind).cuda())

        def vector(value, size, kind=dtype):
            return torch.nn.Parameter(torch.full((size,), value, dtype=kind, device="cuda"))

        self.norm1_weight, self.norm1_bias = vector(1.0, width), vector(0.0, width)
        self.norm2_weight, self.norm2_bias = vector(1.0, width), vector(0.0, width)
        self.w_in, self.b_in = matrix(self.circuit.num_x, width), vector(0.0, self.circuit.num_x)
        self.angles = torch.nn.Parameter((torch.rand(self.circuit.num_w, generator=g) - 0.5).cuda())
        # the expectations are float32: so is the projection that takes them back
        self.w_out, self.b_out = matrix(width, qubits, torch.float32), vector(0.0, width, torch.float32)
        self.w_gate, self.w_up = matrix(hidden, width), matrix(hidden, width)
        self.w_down = matrix(width, hidden)

    def forward(self, h):
        a = layers.layer_norm(h, self.norm1_weight, self.norm1_bias)
        a = layers.linear(a, self.w_in, self.b_in, "tanh", out_dtype=torch.float32)
        z = self.circuit(a.reshape(-1, self.circuit.num_x), self.angles)
        h = layers.linear(z.reshape(h.shape[:-1] + (self.circuit.n,)), self.w_out, self.b_out, residual=h,
                          out_dtype=h.dtype)
        a = layers.layer_norm(h, self.norm2_weight, self.norm2_bias)
        a = layers.gated(a, self.w_gate, self.w_up)
        return layers.linear(a, self.w_down, residual=h)


class SequenceBlock(_Block):
    """See the module's text.  ``heads`` of ``dim`` elements, ``groups`` of keys and values; ``window`` (None: every
    earlier token) and ``sinks`` first tokens that stay visible; ``dropout`` of the attention's branch in
    training, drawn anew in every forward pass: from torch's generator, or with a ``seed`` of its own from that and the
    count of passes (``draws``)."""
    own_types = ("frequencies",)                  # float64: angles of far positions

    def __init__(self, width: int, heads: int, groups: int, dim: int, qubits: int, window=None, sinks: int = 0,
                 dropout: float = 0.0, dtype=torch.float32, seed: int | None = None, **rest):
        super().__init__()
        self.counts, seed = seed is not None, seed or 0
        self.heads, self.groups, self.dim, self.window, self.sinks, self.dropout = heads, groups, dim, window, sinks, dropout
        g = torch.Generator().manual_seed(seed + 1)

        def matrix(rows, cols):
            return torch.nn.Parameter((torch.randn(rows, cols, generator=g) * cols ** -0.5).to(dtype).cuda())

        def ones(size):
            return torch.nn.Parameter(torch.ones(size, dtype=dtype, device="cuda"))

        self.norm_weight, self.norm_bias = ones(width), torch.nn.Parameter(torch.zeros(width, dtype=dtype, device="cuda"))
        self.w_q, self.w_k, self.w_v = matrix(heads * dim, width), matrix(groups * dim, width), matrix(groups * dim, width)
        self.w_o = matrix(width, heads * dim)
        self.weight_q, self.weight_k = ones(dim), ones(dim)
        self.register_buffer("frequencies", layers.rotary_frequencies(dim))
        self.register_buffer("draws", torch.tensor([seed, 0], device="cuda"))
        self.rest = HybridBlock(width, qubits, dtype=dtype, seed=seed, **rest)

    def _heads(self, h):
        a = layers.layer_norm(h, self.norm_weight, self.norm_bias)
        return [layers.linear(a, w).unflatten(-1, (-1, self.dim)) for w in (self.w_q, self.w_k, self.w_v)]

    def _next_draws(self):
        """Seed and offset of a pass, in a tensor of their own: its backward draws the same elements again.  (Torch's generator
        is put back for a pass that is made again, and goes on in the replays of a captured one.)"""
        if not self.counts:
            return torch.empty_like(self.draws).random_()
        if torch._C._current_graph_task_id() >= 0:      # inside of a backward pass
            raise RuntimeError("a forward pass that is made again for its backward (activation checkpointing) would draw other "
                               "elements than the first one: give the block its draws, or no seed")
        draws = self.draws.clone()
        self.draws[1] += 1
        return draws

    def forward(self, h, lengths=None, draws=None):
        """``draws``: seed and offset of the dropout, an int64 tensor on the device, in the place of the block's own."""
        q, k, v = self._heads(h)
        q, k = layers.norm_rotary(q, k, self.weight_q, self.weight_k, self.frequencies)
        a = layers.attention(q, k, v, self.window, self.sinks, lengths=lengths).flatten(-2)
        if self.training and self.dropout:
            h = layers.dropout(layers.linear(a, self.w_o), self.dropout, self._next_draws() if draws is None else draws, residual=h)
        else:
            h = layers.linear(a, self.w_o, residual=h)
        return self.rest(h)

    def cache(self, batch, capacity):
        """Keys and values of ``capacity`` tokens of each sequence."""
        shape = (2, batch, capacity, self.groups, self.dim)
        return torch.zeros(shape, dtype=self.w_q.dtype, device=self.w_q.device)

    @torch.no_grad()
    def step(self, h, cache, lengths):
        """The next tokens h [batch, tokens, width] of sequences; lengths (int32 [batch]) counts them in."""
        q, k, v = self._heads(h)
        q = layers.norm_rotary_step(q, k, v, cache[0], cache[1], lengths, self.weight_q, self.weight_k, self.frequencies)
        a = layers.attention_step(q, cache[0], cache[1], lengths, self.window, self.sinks).flatten(-2)
        return self.rest(layers.linear(a, self.w_o, residual=h))


def train_sequence(width=256, qubits=6, batch=16, tokens=64, steps=40, rate=0.02, dtype=torch.bfloat16, seed=0, window=16,
                   sinks=2, dropout=0.1, say=print):
    """Losses of ``steps`` steps on a synthetic task over sequences: a token's first feature is to follow the
    product of two features of the token before it."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = SequenceBlock(width, 4, 2, 64, qubits, window, sinks, dropout, dtype, seed)
    opt = torch.optim.SGD(block.parameters(), lr=rate, momentum=0.9)
    x = torch.randn(batch, tokens, width, generator=g, device="cuda")
    target = torch.tanh(x[:, :-1, 1] * x[:, :-1, 2])
    x = x.to(dtype)
    losses = []
    for step in range(steps):
        loss = (block(x)[:, 1:, 0].float() - target).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    losses = [float(v) for v in losses]
    B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)
    for step in sorted(set(range(0, steps, max(1, steps // 8))) | {steps - 1}):
        say("step %3d  loss %.4f" % (step, losses[step]))
    return losses


def train(width=256, qubits=6, batch=512, steps=40, rate=0.02, dtype=torch.bfloat16, seed=0, say=print):
    """Losses of ``steps`` steps of gradient descent (momentum 0.9) on a synthetic
    regression: the block's first feature is to follow a product of two others."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block = HybridBlock(width, qubits, dtype=dtype, seed=seed)
    opt = torch.optim.SGD(block.parameters(), lr=rate, momentum=0.9)
    x = torch.randn(batch, width, generator=g, device="cuda")
    target = torch.tanh(x[:, 1] * x[:, 2])
    x = x.to(dtype)
    losses = []
    for step in range(steps):
        loss = (block(x)[:, 0].float() - target).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    losses = [float(v) for v in losses]
    B.vqc_sync_check(torch.cuda.current_stream().cuda_stream)
    for step in range(0, steps, max(1, steps // 8)):
        say("step %3d  loss %.4f" % (step, losses[step]))
    say("step %3d  loss %.4f" % (steps - 1, losses[-1]))
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--qubits", type=int, default=6)
    ap.add_argument("--batch", type=int, default=512)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--dtype", choices=("float32", "bfloat16", "float16"), default="bfloat16")
    ap.add_argument("--tokens", type=int, default=0, help="tokens of a sequence: train a sequence block")
    ap.add_argument("--window", type=int, default=16)
    a = ap.parse_args()
    if a.tokens:
        train_sequence(a.width, a.qubits, max(1, a.batch // a.tokens), a.tokens, a.steps, dtype=getattr(torch, a.dtype),
                       window=a.window)
    else:
        train(a.width, a.qubits, a.batch, a.steps, dtype=getattr(torch, a.dtype))


if __name__ == "__main__":
    main()
