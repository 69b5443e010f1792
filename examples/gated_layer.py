"""Trains a gated layer (d = 256: Wq, Wo of 256 x 256, Wk, Wv of 128 x 256, gate and up of 1024 x 256, down of 256 x 1024) with activations in 8 bits.

RMS norm, rotary positions and attention with shared key heads come from `paper_2609_21594_b200.functional`, as do the projections, whose products are
formed in 8 bits, and the gated feed-forward block, which keeps x, gate and up in 8 bits for its backward pass (`--full`: both in bf16).  The
seven matrices are updated by `paper_2609_21594_b200.optim.Muon`, everything else by torch's AdamW.  The documents are those of tiny_layer.py.

    python examples/gated_layer.py --steps 200
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2609_21594_b200 import functional as F  # noqa: E402
from paper_2609_21594_b200.optim import Muon  # noqa: E402
from tiny_layer import VOCAB, batch  # noqa: E402

DIM, HEADS, KV_HEADS, HIDDEN = 256, 4, 2, 1024
HEAD = DIM // HEADS


class GatedLayer(torch.nn.Module):
    """Embedding, one pre-norm layer, norm, output.  Parameters are fp32, the layer computes in bf16."""

    def __init__(self, generator: torch.Generator, eight: bool = True):
        super().__init__()
        matrix = lambda rows, cols: torch.nn.Parameter(torch.randn((rows, cols), generator=generator, device="cuda") * cols ** -0.5)  # noqa: E731
        self.eight = eight
        self.embedding = torch.nn.Parameter(torch.randn((VOCAB, DIM), generator=generator, device="cuda") * DIM ** -0.5)
        self.wq, self.wk, self.wv, self.wo = matrix(DIM, DIM), matrix(KV_HEADS * HEAD, DIM), matrix(KV_HEADS * HEAD, DIM), matrix(DIM, DIM)
        self.gate, self.up, self.down = matrix(HIDDEN, DIM), matrix(HIDDEN, DIM), matrix(DIM, HIDDEN)
        self.norms = torch.nn.ParameterList([torch.nn.Parameter(torch.ones(DIM, device="cuda")) for _ in range(3)])
        self.inv_freq = F.rotary_frequencies(10000.0, HEAD)

    def matrices(self):
        return [self.wq, self.wk, self.wv, self.wo, self.gate, self.up, self.down]

    def others(self):
        return [self.embedding, *self.norms]

    def forward(self, tokens: torch.Tensor, positions: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        """tokens, positions: [n]; offsets: where the documents begin and end.  Logits [n, vocabulary]."""
        norm = lambda x, i: F.layer_norm(x, self.norms[i], center=False)  # noqa: E731
        half = lambda w: w.to(torch.bfloat16)  # noqa: E731
        times = F.linear_8bit if self.eight else lambda x, w: x @ half(w).T
        x = half(self.embedding)[tokens]
        h = norm(x, 0)
        q, k, v = (times(h, w).view(len(tokens), -1, HEAD) for w in (self.wq, self.wk, self.wv))
        q, k = F.rotary((q, k), self.inv_freq, positions=positions)
        a = F.attention(q, k, v, causal=True, q_offsets=offsets, k_offsets=offsets)
        x = x + times(a.reshape(-1, DIM), self.wo)
        x = x + F.feed_forward(norm(x, 1), half(self.gate), half(self.up), half(self.down), checkpoint="8bit" if self.eight else "full")
        return (norm(x, 2) @ half(self.embedding).T).float()


def train(steps: int, seed: int = 0, report: int = 0, eight: bool = True):
    """Losses (in nats per token) of `steps` steps."""
    generator = torch.Generator(device="cuda").manual_seed(seed)
    model = GatedLayer(generator, eight)
    muon = Muon(model.matrices(), lr=0.02, momentum=0.95)
    adam = torch.optim.AdamW(model.others(), lr=3e-3, weight_decay=0.0)
    losses = []
    for step in range(steps):
        tokens, positions, offsets, learn = batch(generator)
        logits = model(tokens, positions, offsets)
        loss = torch.nn.functional.cross_entropy(logits[learn], tokens[learn + 1])
        muon.zero_grad()
        adam.zero_grad()
        loss.backward()
        muon.step()
        adam.step()
        losses.append(loss.detach())
        if report and (step + 1) % report == 0:
            print(f"step {step + 1:4d}  loss {float(losses[-1]):.3f}", flush=True)
    F.synchronize_and_check()                            # no bounded wait has expired, in the backward passes' thread either
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=200)
    parser.add_argument("--seed", type=int, default=0)
    parser.add_argument("--full", action="store_true")
    args = parser.parse_args()
    train(args.steps, args.seed, report=max(1, args.steps // 10), eight=not args.full)
