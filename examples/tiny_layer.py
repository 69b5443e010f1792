"""Trains the tiny layer (d = 256: Wq, Wk, Wv, Wo of 256 x 256, W_up 1024 x 256, W_down 256 x 1024) end to end with the framework's operators.

Layer norm, rotary positions and attention (documents of uneven lengths packed into one row) come from
`paper_2609_21594_b200.functional`; the six matrices are updated by `paper_2609_21594_b200.optim.Muon`, everything else by torch's AdamW.  Every
document repeats a pattern of its own with a period of eight tokens, so the loss falls once attention finds the token eight back.

    python examples/tiny_layer.py --steps 200
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_21594_b200 import functional as F  # noqa: E402
from paper_2609_21594_b200.optim import Muon  # noqa: E402

DIM, HEADS, VOCAB, PERIOD = 256, 4, 64, 8


class TinyLayer(torch.nn.Module):
    """Embedding, one pre-norm transformer layer, norm, output.  Parameters are fp32, the layer computes in bf16."""

    def __init__(self, generator: torch.Generator):
        super().__init__()
        matrix = lambda rows, cols: torch.nn.Parameter(torch.randn((rows, cols), generator=generator, device="cuda") * cols ** -0.5)  # noqa: E731
        self.embedding = torch.nn.Parameter(torch.randn((VOCAB, DIM), generator=generator, device="cuda") * DIM ** -0.5)
        self.wq, self.wk, self.wv, self.wo = (matrix(DIM, DIM) for _ in range(4))
        self.up, self.down = matrix(4 * DIM, DIM), matrix(DIM, 4 * DIM)
        self.norms = torch.nn.ParameterList([torch.nn.Parameter(torch.ones(DIM, device="cuda")) for _ in range(3)])
        self.biases = torch.nn.ParameterList([torch.nn.Parameter(torch.zeros(DIM, device="cuda")) for _ in range(3)])
        self.inv_freq = F.rotary_frequencies(10000.0, DIM // HEADS)

    def matrices(self):
        return [self.wq, self.wk, self.wv, self.wo, self.up, self.down]

    def others(self):
        return [self.embedding, *self.norms, *self.biases]

    def forward(self, tokens: torch.Tensor, positions: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        """tokens, positions: [n]; offsets: where the documents begin and end.  Logits [n, vocabulary]."""
        norm = lambda x, i: F.layer_norm(x, self.norms[i], self.biases[i])  # noqa: E731
        times = lambda x, w: x @ w.to(torch.bfloat16).T  # noqa: E731
        x = self.embedding.to(torch.bfloat16)[tokens]
        h = norm(x, 0)
        q, k, v = (times(h, w).view(-1, HEADS, DIM // HEADS) for w in (self.wq, self.wk, self.wv))
        q, k = F.rotary((q, k), self.inv_freq, positions=positions)
        a = F.attention(q, k, v, causal=True, q_offsets=offsets, k_offsets=offsets)
        x = x + times(a.reshape(-1, DIM), self.wo)
        x = x + times(torch.relu(times(norm(x, 1), self.up)), self.down)
        return times(norm(x, 2), self.embedding).float()


def batch(generator: torch.Generator, documents: int = 12):
    """Documents of 40 to 200 tokens in one row: tokens, positions inside the documents, offsets, and which tokens have a successor to learn."""
    lengths = torch.randint(40, 201, (documents,), generator=generator, device="cuda")
    offsets = torch.cat([lengths.new_zeros(1), lengths.cumsum(0)])
    i = torch.arange(int(offsets[-1]), device="cuda")
    doc = (i[:, None] >= offsets[None, 1:]).sum(-1)
    positions = i - offsets[doc]
    patterns = torch.randint(0, VOCAB, (documents, PERIOD), generator=generator, device="cuda")
    tokens = patterns[doc, positions % PERIOD]
    learn = torch.nonzero((positions >= PERIOD) & (positions < lengths[doc] - 1)).squeeze(-1)
    return tokens, positions.to(torch.int32), offsets.to(torch.int32), learn


def train(steps: int, seed: int = 0, report: int = 0):
    """Losses (in nats per token) of `steps` steps."""
    generator = torch.Generator(device="cuda").manual_seed(seed)
    model = TinyLayer(generator)
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
    args = parser.parse_args()
    train(args.steps, args.seed, report=max(1, args.steps // 10))
