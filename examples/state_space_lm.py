#!/usr/bin/env python
"""A small state space language model on the operator library: training steps and token-by-token decoding.

  one-hot tokens -> dense (embedding) -> dense -> short convolution -> dense (steps) and dense (input and output weights)
                 -> selective scan, gated by another dense of the embedding -> dense -> log-probabilities of the next tokens

The head is the embedding table itself, and the scores of a training step are never stored: the log-probabilities come straight from the
head's operands.  Training runs the groups backwards (Section 4.2 of the paper: the gradient program is a program like any other) and
applies the partials with the SGD update.  Decoding feeds one token at a time to the same convolution and scan (T = 1) and carries
their states on.  All arithmetic is the library's; torch holds the memory.

  python examples/state_space_lm.py [--steps N]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_1810_00952_b200 import binding as B  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32
ADD = dict(op=[0], a=[0], b=[1], c=[-1], dtype=[B.BF16], imm=[0.0])                          # x0 + x1
ADD3 = dict(op=[0, 0], a=[0, 3], b=[1, 2], c=[-1, -1], dtype=[B.BF16] * 2, imm=[0.0] * 2)    # x0 + x1 + x2


class StateSpaceLM:
    """Weights, the buffers of one batch shape, and the calls of a step."""

    def __init__(self, vocabulary: int, width: int, inner: int, states: int, steps: int, batch: int, taps: int = 4, seed: int = 0,
                 device="cuda:0"):
        g = torch.Generator(device=device).manual_seed(seed)
        V, D, E, N, T, Bn = vocabulary, width, inner, states, steps, batch
        self.V, self.D, self.E, self.N, self.T, self.Bn, self.K, self.device = V, D, E, N, T, Bn, taps, device

        def weight(rows, cols, scale=1.0):
            return (scale * torch.randn(rows, cols, generator=g, device=device) / rows ** 0.5).to(BF16)

        # bf16: embedding and head, the layer's dense weights; f32: filter and bias, decays, skip, bias of the steps
        self.weights = dict(table=weight(V, D, 0.2 * V ** 0.5), w_x=weight(D, E), w_z=weight(D, E), w_step=weight(E, E, 0.3), w_bc=weight(E, 2 * N),
                            w_out=weight(E, D))
        self.weights.update(w_conv=torch.randn(taps, E, generator=g, device=device) / taps ** 0.5, b_conv=torch.zeros(E, device=device),
                            a=-torch.arange(1.0, N + 1, device=device).repeat(E, 1), skip=torch.ones(E, device=device),
                            b_step=torch.full((E,), -3.0, device=device))
        self.partials = {k: torch.empty_like(w) for k, w in self.weights.items()}

        def buf(*shape, dtype=BF16):
            return torch.empty(shape, dtype=dtype, device=device)

        for k, n in dict(e=D, x=E, z=E, u=E, step=E, bc=2 * N, y=E, h=D).items():
            setattr(self, k, buf(T, Bn, n))
            setattr(self, "d" + k, buf(T, Bn, n))
        self.du2, self.du3, self.de2 = buf(T, Bn, E), buf(T, Bn, E), buf(T, Bn, D)
        self.table1, self.table2 = buf(V, D), buf(V, D)
        self.states = buf(-(-T // B.SCAN_SPAN), Bn, E, N, dtype=F32)
        self.logp, self.lse = buf(T, Bn, dtype=F32), buf(T, Bn, dtype=F32)
        w = self.weights
        dense = [(buf(T, Bn, V), w["table"]), (self.e, w["w_x"]), (self.u, w["w_step"]), (self.u, w["w_bc"]), (self.y, w["w_out"])]
        self.ws = buf(max([16, B.relay_workspace_bytes_causal_conv_grad(self.x, w["w_conv"]), B.relay_workspace_bytes_selective_scan_grad(self.u, w["a"]),
                           B.relay_workspace_bytes_linear_logprob(self.h, w["table"], True),
                           B.relay_workspace_bytes_linear_logprob_grad(self.h, w["table"], True)] +
                          [B.relay_workspace_bytes_dense_act_grad(x, v) for x, v in dense]), dtype=torch.uint8)

    def one_hot(self, tokens: torch.Tensor) -> torch.Tensor:
        return torch.nn.functional.one_hot(tokens.long(), self.V).to(BF16)

    def dense(self, x, name, y):
        B.relay_fused_dense_act(x, self.weights[name], None, B.ACT_NONE, y, self.ws)

    def dense_grad(self, x, name, y, dy, dx, dw=None):
        B.relay_fused_dense_act_grad(x, self.weights[name], y, dy, B.ACT_NONE, dx, self.partials[name] if dw is None else dw, None, self.ws)

    def forward(self, x: torch.Tensor, targets: torch.Tensor, lengths=None) -> torch.Tensor:
        """x (T,B,V) one-hot, targets (T,B): the next tokens, -1 where there is none -> their log-probabilities (T,B)."""
        w = self.weights
        self.dense(x, "table", self.e)
        self.dense(self.e, "w_x", self.x)
        self.dense(self.e, "w_z", self.z)
        B.relay_causal_conv(self.x, w["w_conv"], w["b_conv"], None, lengths, B.ACT_SILU, self.u, None)
        self.dense(self.u, "w_step", self.step)
        self.dense(self.u, "w_bc", self.bc)
        B.relay_selective_scan(self.u, self.step, w["a"], self.bc, None, w["skip"], self.z, w["b_step"], None, lengths, True, self.y, None, self.states)
        self.dense(self.y, "w_out", self.h)
        B.relay_linear_logprob(self.h, w["table"], True, targets, 1.0, self.logp, self.lse, self.ws)
        return self.logp

    def backward(self, x: torch.Tensor, targets: torch.Tensor, dlogp: torch.Tensor, lengths=None):
        """Partials of all weights, given those of the log-probabilities; `forward` ran on the same batch."""
        w, p = self.weights, self.partials
        B.relay_linear_logprob_grad(self.h, w["table"], True, targets, 1.0, self.lse, dlogp, self.dh, self.table1, self.ws)
        self.dense_grad(self.y, "w_out", self.h, self.dh, self.dy)
        B.relay_selective_scan_grad(self.u, self.step, w["a"], self.bc, None, w["skip"], self.z, w["b_step"], lengths, True, self.states, self.dy, None,
                                    self.du, self.dstep, p["a"], self.dbc, None, p["skip"], self.dz, p["b_step"], None, self.ws)
        self.dense_grad(self.u, "w_step", self.step, self.dstep, self.du2)
        self.dense_grad(self.u, "w_bc", self.bc, self.dbc, self.du3)
        B.relay_fused_ewise(ADD3, [self.du, self.du2, self.du3], [4], [self.dy])             # all that flows back into u
        B.relay_causal_conv_grad(self.x, w["w_conv"], w["b_conv"], None, lengths, B.ACT_SILU, self.dy, None, self.dx, p["w_conv"], p["b_conv"], None,
                                 self.ws)
        self.dense_grad(self.e, "w_x", self.x, self.dx, self.de)
        self.dense_grad(self.e, "w_z", self.z, self.dz, self.de2)
        B.relay_fused_ewise(ADD, [self.de, self.de2], [2], [self.dh])
        self.dense_grad(x, "table", self.e, self.dh, None, self.table2)
        B.relay_fused_ewise(ADD, [self.table1, self.table2], [2], [p["table"]])                 # the table is used twice: its partials add up

    def train_step(self, tokens: torch.Tensor, lr: float) -> torch.Tensor:
        """tokens (T+1,B) i32 -> log-probabilities of tokens[1:] before the step (T,B)."""
        x, targets = self.one_hot(tokens[:-1]), tokens[1:].clone()
        logp = self.forward(x, targets).clone()
        self.backward(x, targets, torch.full_like(logp, -1.0 / logp.numel()))                # of the mean negative log-probability
        names = list(self.weights)
        B.relay_sgd_update([self.weights[k] for k in names], [self.partials[k] for k in names], lr)
        return logp

    def decode(self, prompt: torch.Tensor, steps: int, top: int = 4):
        """prompt (T0,B) i32 -> the most probable continuation (steps,B) and the alternatives' log-probabilities (steps,B,top)."""
        w, n, dev = self.weights, prompt.shape[1], self.device

        def row(width):
            return torch.empty(1, n, width, dtype=BF16, device=dev)

        e, x, z, u, step, bc, y, h, scores = (row(k) for k in (self.D, self.E, self.E, self.E, self.E, 2 * self.N, self.E, self.D, self.V))
        taps, taps2 = (torch.zeros(self.K - 1, n, self.E, dtype=BF16, device=dev) for _ in range(2))
        state, state2 = (torch.zeros(n, self.E, self.N, device=dev) for _ in range(2))
        ids, alternatives = torch.empty(1, n, top, dtype=torch.int32, device=dev), torch.empty(1, n, top, device=dev)
        out, logs = [], []
        for k in range(prompt.shape[0] + steps - 1):
            token = prompt[k] if k < prompt.shape[0] else out[-1]
            self.dense(self.one_hot(token)[None], "table", e)
            self.dense(e, "w_x", x)
            self.dense(e, "w_z", z)
            B.relay_causal_conv(x, w["w_conv"], w["b_conv"], taps, None, B.ACT_SILU, u, taps2)
            self.dense(u, "w_step", step)
            self.dense(u, "w_bc", bc)
            B.relay_selective_scan(u, step, w["a"], bc, None, w["skip"], z, w["b_step"], state, None, True, y, state2, None)
            taps, taps2, state, state2 = taps2, taps, state2, state
            if k + 1 < prompt.shape[0]:
                continue
            self.dense(y, "w_out", h)
            B.relay_contract_act(h[0], 0, w["table"], 1, None, B.ACT_NONE, scores[0])
            B.relay_token_logprob(scores, None, 1.0, None, None, None, alternatives, ids)
            out.append(ids[0, :, 0].clone())
            logs.append(alternatives[0].clone())
        return torch.stack(out), torch.stack(logs)


def patterns(T: int, n: int, V: int, seed: int, device="cuda:0") -> torch.Tensor:
    """(T,n) tokens: each sequence repeats a random pattern of five distinct tokens."""
    g = torch.Generator().manual_seed(seed)
    motif = torch.stack([torch.randperm(V, generator=g)[:5] for _ in range(n)], dim=1)
    return motif[torch.arange(T) % 5].to(torch.int32).to(device)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=400)
    ap.add_argument("--lr", type=float, default=1.0)
    a = ap.parse_args()
    model = StateSpaceLM(vocabulary=64, width=64, inner=128, states=16, steps=63, batch=16)
    tokens = patterns(64, 16, 64, 1)
    for k in range(a.steps):
        logp = model.train_step(tokens, a.lr)
        if k % max(1, a.steps // 10) == 0:
            print(f"step {k:4d}  mean log-probability {float(logp.mean()):8.4f}")
    said, logs = model.decode(tokens[:10], 20)
    print("continuation as seen in training:", bool(torch.equal(said, tokens[10:30])),
          " mean log-probability of the best alternative:", round(float(logs[..., 0].mean()), 4))
    B.relay_poll_status()


if __name__ == "__main__":
    main()
