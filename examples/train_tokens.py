"""Next-token training of a one-layer dendritic spiking network, every step in the library.

    ids [T, B] -> embedding: currents and decay gates of every compartment
               -> gated compartment scan over the sequence
               -> DendSN layer (branches, soma, spikes) over the same T steps
               -> linear readout over the vocabulary, softmax cross entropy

The tokens are synthetic: sequences of a random Markov chain in which every token has a few
likely successors, packed end to end, so that a model can learn them and the loss has a known
floor (the chain's entropy).

    python examples/train_tokens.py [--steps 200] [--dtype f32|bf16]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2412_06355_gb300 import (DendSNFunction, EmbedFunction, ScanFunction,  # noqa: E402
                                    XentFunction, make_config)


class TokenModel(torch.nn.Module):
    """V tokens, N dendritic neurons of K compartments."""

    def __init__(self, V, N, K, T, B, dtype=torch.float32, device="cuda"):
        super().__init__()
        name = "bf16" if dtype == torch.bfloat16 else "f32"
        self.shape = (T, B, N, K)
        self.cfg = make_config(T, B, N, K, G=1, C=N, inner=1, dtype=name, beta=0.5)

        def parameter(t):
            return torch.nn.Parameter(t.to(device))

        self.currents = parameter(torch.randn(V, N * K).to(dtype))
        self.gates = parameter((torch.randn(V, N * K) * 0.5).to(dtype))
        self.alpha = parameter(torch.full((N, K), 0.5))
        self.xi = parameter(torch.randn(N, K) * 0.1)
        self.zeta = parameter(torch.ones(N, K))
        self.kappa = parameter(torch.full((N, K), 1.5 / K) + torch.randn(N, K) * 0.3)
        self.readout = parameter((torch.randn(V, N) / math.sqrt(N)).to(dtype))

    def forward(self, ids, starts, labels):
        """Row losses [T * B] of predicting labels [T, B] (negative: not counted)."""
        T, B, N, K = self.shape
        x = EmbedFunction.apply(self.currents, ids)
        gate = EmbedFunction.apply(self.gates, ids)
        h, _ = ScanFunction.apply(x, gate, starts, None, "logit", "complement")
        spikes = DendSNFunction.apply(h.view(T, B, N, K), self.alpha, self.xi, self.zeta,
                                      self.kappa, None, self.cfg)
        return XentFunction.apply(spikes.view(T * B, N), self.readout, labels.reshape(-1), -1)


class MarkovTokens:
    """Sequences of a random chain with `fan` successors of each token, packed end to end."""

    def __init__(self, V, fan=4, seed=0, device="cuda"):
        self.g = torch.Generator(device=device)
        self.g.manual_seed(seed)
        self.V, self.device = V, device
        self.next = torch.randint(0, V, (V, fan), generator=self.g, device=device)
        self.prob = torch.softmax(torch.randn(V, fan, generator=self.g, device=device), 1)

    def entropy(self):
        p = torch.zeros(self.V, self.V, device=self.device).scatter_add_(1, self.next, self.prob)
        return float(-(p * p.clamp_min(1e-30).log()).sum(1).mean())

    def batch(self, T, B, new=0.02):
        """(ids, starts, labels) [T, B]; the last token of a sequence predicts nothing."""
        ids = torch.empty(T + 1, B, dtype=torch.int64, device=self.device)
        first = torch.rand(T + 1, B, generator=self.g, device=self.device) < new
        first[0] = True
        fresh = torch.randint(0, self.V, (T + 1, B), generator=self.g, device=self.device)
        u = torch.rand(T + 1, B, 1, generator=self.g, device=self.device)
        for t in range(T + 1):
            if t:
                pick = (u[t] > self.prob[ids[t - 1]].cumsum(1)).sum(1).clamp_max(self.next.shape[1] - 1)
                ids[t] = torch.where(first[t], fresh[t], self.next[ids[t - 1], pick])
            else:
                ids[t] = fresh[t]
        labels = torch.where(first[1:], torch.full_like(ids[1:], -1), ids[1:])
        return ids[:T].contiguous(), first[:T].to(torch.uint8), labels


def train(steps=200, V=512, N=256, K=4, T=64, B=32, dtype=torch.float32, lr=0.02, seed=0, report=None):
    """Trains and returns the mean loss of every step."""
    torch.manual_seed(seed)
    data = MarkovTokens(V, seed=seed)
    model = TokenModel(V, N, K, T, B, dtype)
    opt = torch.optim.Adam(model.parameters(), lr=lr)
    losses = []
    for step in range(steps):
        ids, starts, labels = data.batch(T, B)
        rows = model(ids, starts, labels)
        loss = rows.sum() / (labels >= 0).sum()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        with torch.no_grad():
            model.zeta.clamp_min_(0.1)
            model.alpha.clamp_(0.0, 0.99)
        losses.append(loss.detach())
        if report and step % report == 0:
            print(f"step {step:4d}  loss {float(losses[-1]):.4f}")
    if report:
        print(f"last 10 steps: {float(torch.stack(losses[-10:]).mean()):.4f}   "
              f"(uniform {math.log(V):.4f}, chain entropy {data.entropy():.4f})")
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args()
    train(a.steps, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32, report=20)
