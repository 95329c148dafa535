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

``python -m paper_2607_11985_gb300.hybrid`` trains one block on a synthetic task.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B, layers, workloads as wl
from .circuit import Circuit


class HybridBlock(torch.nn.Module):
    """See the module's text.  ``spec``: a circuit with one x angle per qubit
    (``workloads.CircuitSpec``), by default a layered ansatz of RY, RZ and CX."""

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
    a = ap.parse_args()
    train(a.width, a.qubits, a.batch, a.steps, dtype=getattr(torch, a.dtype))


if __name__ == "__main__":
    main()
