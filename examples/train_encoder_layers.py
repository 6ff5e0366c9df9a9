"""A query encoder of layers trained from the retrieval it drives: the operators of hr_layers.h between a search and its loss.

    python examples/train_encoder_layers.py [--passages N] [--steps S] [--layers L]

The loop of teach_query_encoder.py with an encoder in the place of a matrix.  A layer is x + gated(norm(x)) w_down': layer norm
(layer_norm), the gated half of a feed-forward block (gated, keep=True) and a plain product.  Every step searches the index with the
encoded questions (IvfIndex.search), lets a reader score what came back, takes the loss over the whole corpus and its gradient at the scores
(i8_linear, distill_step), takes that back through the layers (gated_backward, layer_norm_backward), last layer first, and updates all
tensors in one call (adamw): matrices in bfloat16 with masters in 32 bits and moments in 8, norms in float32.

Synthetic data, as there: a question is a passage seen through noise and a rotation that the encoder has to undo.
"""
import argparse
import importlib.util
import math
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(HERE))
import paper_2507_09138_amd as hr  # noqa: E402

_spec = importlib.util.spec_from_file_location("teach_query_encoder", os.path.join(HERE, "teach_query_encoder.py"))
data = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(data)
SCALE = data.SCALE


class Encoder:
    """Layers over rows of d numbers, and what updates them.  Tensors by layer: norm's weight and bias, w_gate, w_up, w_down."""

    def __init__(self, layers, d, hidden, dtype=torch.bfloat16, bits=8, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.tensors = []
        for _ in range(layers):
            self.tensors += [torch.ones(d, device="cuda"), torch.zeros(d, device="cuda")]
            for rows, cols in ((hidden, d), (hidden, d), (d, hidden)):
                self.tensors.append((torch.randn(rows, cols, generator=g, device="cuda") / math.sqrt(cols)).to(dtype))
        self.masters = [None if t.dtype == torch.float32 else t.float() for t in self.tensors]
        state = [hr.adamw_state(t, bits if t.dim() == 2 else 32) for t in self.tensors]
        self.m, self.v, self.exponents = ([s[i] for s in state] for i in range(3))
        self.decay = [0.01 if t.dim() == 2 else 0.0 for t in self.tensors]
        self.dtype, self.steps = dtype, 0

    def layers(self):
        return [self.tensors[i:i + 5] for i in range(0, len(self.tensors), 5)]

    def forward(self, x):
        """Rows through all layers: what comes out, and what ``backward`` needs."""
        x, kept = x.to(self.dtype), []
        for weight, bias, w_gate, w_up, w_down in self.layers():
            normed = hr.layer_norm(x, weight, bias)
            h = hr.gated(normed.out, w_gate, w_up, keep=True)
            kept.append((x, normed, h))
            x = x + h.out @ w_down.T
        return x, kept

    def backward(self, grad, kept):
        """Gradients of all tensors, in their order, from that of the rows that came out."""
        found, grad = [], grad.to(self.dtype)
        for (weight, bias, w_gate, w_up, w_down), (x, normed, h) in zip(reversed(self.layers()), reversed(kept)):
            grad_down = grad.T @ h.out
            gates = hr.gated_backward(normed.out, w_gate, w_up, h.pre, grad @ w_down)
            norms = hr.layer_norm_backward(x, weight, normed.stats, gates.x)
            grad = grad + norms.x
            found = [norms.weight, norms.bias, gates.w_gate, gates.w_up, grad_down] + found
        return found

    def step(self, grads, rate):
        self.steps += 1
        hr.adamw(self.tensors, grads, self.m, self.v, self.steps, rate, weight_decay=self.decay, exponents=self.exponents, masters=self.masters)


def encode(encoder, seen):
    """Unit vectors to search with, and what the gradient needs."""
    raw, kept = encoder.forward(seen)
    raw = raw.float()
    norm = raw.norm(dim=1, keepdim=True)
    return raw / norm, norm, kept


def main(passages=65536, d=256, hidden=512, layers=2, nlist=256, batch=512, k=32, probes=8, steps=200, rate=2e-3, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ix, rows = data.corpus(passages, d, nlist, g)
    rows8, scale8 = hr.quantize_rows(rows)
    skew = torch.randn(d, d, generator=g, device="cuda")
    turn = torch.matrix_exp(1.35 * (skew - skew.T) / (2 * d) ** 0.5)
    encoder = Encoder(layers, d, hidden, seed=seed)
    weights = torch.full((batch,), 1.0 / batch, device="cuda")
    losses = []
    for step in range(steps):
        seen, clean, gold = data.questions(rows, batch, turn, g)
        q, norm, kept = encode(encoder, seen * math.sqrt(d))
        ids, _ = ix.search(q, probes, k)
        reader = (rows[ids.clamp(min=0)] * clean[:, None, :]).sum(2)
        scores = hr.i8_linear(q, rows8, scale8)
        loss, grad = hr.distill_step(scores, ids, reader, weights, scale=SCALE, out=scores)
        dq = grad @ rows
        encoder.step(encoder.backward((dq - q * (dq * q).sum(1, keepdim=True)) / norm, kept), rate)
        losses.append(loss.mean())
        if step % 20 == 0 or step == steps - 1:
            r = hr.logprobs(hr.i8_linear(q, rows8, scale8), gold, scale=SCALE)
            print(f"step {step}: loss {float(losses[-1]):.4f}, ln p of the right passage {float(r.logprobs.mean()):.3f}", flush=True)
    ix.close()
    return encoder, [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--passages", type=int, default=65536)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    main(passages=a.passages, steps=a.steps, layers=a.layers)
