#!/usr/bin/env python
"""A small recurrent language model on the operator library: training steps and token-by-token decoding.

  one-hot tokens -> dense (embedding) -> dense (gates | values) -> gated linear recurrence -> dense (scores)
                 -> log-probabilities of the next tokens

Training runs the groups backwards (Section 4.2 of the paper: the gradient program is a program like any other), orthogonalises the
partials of the weight matrices and applies them with the SGD update.  Decoding feeds one token at a time to the same recurrence
call (T = 1) and reads the most probable alternatives off the scores.  All arithmetic is the library's; torch holds the memory.

  python examples/recurrent_lm.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_1810_00952_b200 import binding as B  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
QUINTIC = (3.4445, -4.7750, 2.0315)


class RecurrentLM:
    """Weights (bf16), the buffers of one batch shape, and the calls of a step."""

    def __init__(self, vocabulary: int, width: int, steps: int, batch: int, seed: int = 0, device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device=device) / rows ** 0.5).to(BF16)

        self.V, self.D, self.T, self.N, self.device = vocabulary, width, steps, batch, device
        self.weights = [weight(vocabulary, width), weight(width, 2 * width), weight(width, vocabulary)]
        T, N, D, V = steps, batch, width, vocabulary

        def buf(*shape, dtype=BF16):
            return torch.empty(shape, dtype=dtype, device=device)

        self.h0 = torch.zeros(N, D, device=device)
        self.e, self.z, self.h, self.scores = buf(T, N, D), buf(T, N, 2 * D), buf(T, N, D), buf(T, N, V)
        self.logp, self.entropy, self.lse = (buf(T, N, dtype=F32) for _ in range(3))
        self.dscores, self.dh, self.dz, self.de = buf(T, N, V), buf(T, N, D), buf(T, N, 2 * D), buf(T, N, D)
        self.partials = [torch.empty_like(w) for w in self.weights]
        self.updates = [torch.empty_like(w) for w in self.weights]
        self.ws = buf(max([16] + [B.relay_workspace_bytes_dense_act_grad(x, w) for x, w in zip((self.scores, self.e, self.h), self.weights)] +
                          [B.relay_workspace_bytes_orthogonalize(w) for w in self.weights]), dtype=torch.uint8)

    def one_hot(self, tokens: torch.Tensor) -> torch.Tensor:
        return torch.nn.functional.one_hot(tokens.long(), self.V).to(BF16)

    def forward(self, x: torch.Tensor, targets: torch.Tensor, lengths=None) -> torch.Tensor:
        """x (T,N,V) one-hot, targets (T,N): the next tokens, -1 where there is none -> their log-probabilities (T,N)."""
        w_e, w_z, w_o = self.weights
        B.relay_fused_dense_act(x, w_e, None, B.ACT_NONE, self.e, self.ws)
        B.relay_fused_dense_act(self.e, w_z, None, B.ACT_NONE, self.z, self.ws)
        B.relay_gated_recurrence(self.z, None, self.h0, lengths, B.GATE_MIX, self.h, None)
        B.relay_fused_dense_act(self.h, w_o, None, B.ACT_NONE, self.scores, self.ws)
        B.relay_token_logprob(self.scores, targets, 1.0, self.logp, self.entropy, self.lse)
        return self.logp

    def backward(self, x: torch.Tensor, targets: torch.Tensor, dlogp: torch.Tensor, lengths=None):
        """Partials of all weights, given those of the log-probabilities; `forward` ran on the same batch."""
        w_e, w_z, w_o = self.weights
        d_e, d_z, d_o = self.partials
        B.relay_token_logprob_grad(self.scores, targets, 1.0, self.lse, None, dlogp, None, self.dscores)
        B.relay_fused_dense_act_grad(self.h, w_o, self.scores, self.dscores, B.ACT_NONE, self.dh, d_o, None, self.ws)
        B.relay_gated_recurrence_grad(self.z, None, self.h0, lengths, B.GATE_MIX, self.h, self.dh, None, self.dz, None, None)
        B.relay_fused_dense_act_grad(self.e, w_z, self.z, self.dz, B.ACT_NONE, self.de, d_z, None, self.ws)
        B.relay_fused_dense_act_grad(x, w_e, self.e, self.de, B.ACT_NONE, None, d_e, None, self.ws)

    def update(self, lr: float):
        for w, d, u in zip(self.weights, self.partials, self.updates):
            B.relay_orthogonalize(d, 5, QUINTIC, 1e-7, max(1.0, w.shape[0] / w.shape[1]) ** 0.5, u, self.ws)
        B.relay_sgd_update(self.weights, self.updates, lr)

    def train_step(self, tokens: torch.Tensor, lr: float) -> torch.Tensor:
        """tokens (T+1,N) i32 -> mean log-probability of tokens[1:] before the step (a scalar tensor)."""
        x, targets = self.one_hot(tokens[:-1]), tokens[1:].contiguous()
        logp = self.forward(x, targets)
        mean = torch.empty((), device=self.device)
        B.relay_fused_reduce(None, [logp], [(0, B.RED_MEAN, 3, 0)], [mean])
        self.backward(x, targets, torch.full_like(logp, -1.0 / logp.numel()))      # of the mean negative log-probability
        self.update(lr)
        return mean

    def decode(self, prompt: torch.Tensor, steps: int, top: int = 4):
        """prompt (T0,N) i32 -> the most probable continuation (steps,N) and the alternatives' log-probabilities (steps,N,top)."""
        N, D, V, dev = prompt.shape[1], self.D, self.V, self.device
        w_e, w_z, w_o = self.weights
        e, z, h, s = (torch.empty(1, N, n, dtype=BF16, device=dev) for n in (D, 2 * D, D, V))
        state, after = torch.zeros(N, D, device=dev), torch.empty(N, D, device=dev)
        ids, alternatives = torch.empty(1, N, top, dtype=torch.int32, device=dev), torch.empty(1, N, top, device=dev)
        out, logs = [], []
        for k in range(prompt.shape[0] + steps - 1):
            token = prompt[k] if k < prompt.shape[0] else out[-1]
            B.relay_fused_dense_act(self.one_hot(token)[None], w_e, None, B.ACT_NONE, e, self.ws)
            B.relay_fused_dense_act(e, w_z, None, B.ACT_NONE, z, self.ws)
            B.relay_gated_recurrence(z, None, state, None, B.GATE_MIX, h, after)
            state, after = after, state
            if k + 1 < prompt.shape[0]:
                continue
            B.relay_fused_dense_act(h, w_o, None, B.ACT_NONE, s, self.ws)
            B.relay_token_logprob(s, None, 1.0, None, None, None, alternatives, ids)
            out.append(ids[0, :, 0].clone())
            logs.append(alternatives[0].clone())
        return torch.stack(out), torch.stack(logs)


def patterns(T: int, N: int, V: int, seed: int, device="cuda:0") -> torch.Tensor:
    """(T,N) tokens: each sequence repeats a random pattern of five distinct tokens."""
    g = torch.Generator().manual_seed(seed)
    motif = torch.stack([torch.randperm(V, generator=g)[:5] for _ in range(N)], dim=1)
    return motif[torch.arange(T) % 5].to(torch.int32).to(device)


def train(steps: int, vocabulary=64, width=128, length=63, batch=16, lr=0.1, seed=0):
    model = RecurrentLM(vocabulary, width, length, batch, seed)
    tokens = patterns(length + 1, batch, vocabulary, seed + 1)
    return model, tokens, [model.train_step(tokens, lr) for _ in range(steps)]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    model, tokens, means = train(a.steps)
    for k in range(0, a.steps, max(1, a.steps // 10)):
        print(f"step {k:4d}  mean log-probability {float(means[k]):8.4f}")
    said, logs = model.decode(tokens[:10], 20)
    print("continuation as seen in training:", bool(torch.equal(said, tokens[10:30])),
          " mean log-probability of the best alternative:", round(float(logs[..., 0].mean()), 4))
    B.relay_poll_status()


if __name__ == "__main__":
    main()
