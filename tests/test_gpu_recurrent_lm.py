"""The operators of recurrent language models together, as examples/recurrent_lm.py runs them: a training step whose every group is
checked against the oracle on the stored inputs, learning, decoding, stream capture, and the bounds-check build."""
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from oracle import language as L
from paper_1810_00952_b200 import binding as B

from parity import assert_bf16, assert_f32, bf16_ulp, rms, to_np
from test_gpu_bounds_check import child

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

import recurrent_lm as E  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_one_training_step_group_by_group():
    T, N, V, D = 21, 5, 40, 72
    model = E.RecurrentLM(V, D, T, N, seed=3)
    tokens = E.patterns(T + 1, N, V, 4)
    lengths = torch.tensor([21, 13, 1, 0, 20], dtype=torch.int32, device=DEV)
    x, targets = model.one_hot(tokens[:-1]), tokens[1:].clone()
    inside = torch.arange(T, device=DEV)[:, None] < lengths[None, :]
    targets[~inside] = -1                                  # padded positions name no token
    before = [w.clone() for w in model.weights]
    logp = model.forward(x, targets, lengths)
    model.backward(x, targets, torch.full_like(logp, -1.0), lengths)
    model.update(0.5)
    torch.cuda.synchronize()
    B.relay_poll_status()
    w_e, w_z, w_o = (to_np(w) for w in before)
    z, h, scores = to_np(model.z), to_np(model.h), to_np(model.scores)
    n = lengths.tolist()
    want_h, _ = L.gated_recurrence(z[..., :D], z[..., D:], np.zeros((N, D)), n, L.GATE_MIX)
    assert_bf16(model.h, want_h, what="h")
    flat = scores.reshape(T * N, V)
    o = L.token_logprob(flat, to_np(targets).astype(int).reshape(-1), 1.0)
    assert_f32(logp.reshape(-1), o["logp"], what="logp")
    want_ds = L.token_logprob_grad(flat, to_np(targets).astype(int).reshape(-1), 1.0, to_np(model.lse).reshape(-1), None, np.full(T * N, -1.0), None)
    assert_bf16(model.dscores.reshape(T * N, V), want_ds, what="dscores")
    ds = to_np(model.dscores).reshape(T * N, V)
    dh, do, _ = oracle.dense_act_grad(h.reshape(T * N, D), w_o, flat, ds, oracle.ACT_NONE, oracle.BF16, oracle.BF16, oracle.F32)
    assert_bf16(model.dh.reshape(T * N, D), dh, what="dh"); assert_bf16(model.partials[2], do, what="dW_o")
    df, du, _ = L.gated_recurrence_grad(z[..., :D], z[..., D:], np.zeros((N, D)), n, L.GATE_MIX, h, to_np(model.dh), np.zeros((N, D)))
    assert_bf16(model.dz[..., :D], df, what="df"); assert_bf16(model.dz[..., D:], du, what="du")
    assert not bool(model.dz[~inside].any())
    for w0, w1, d, u in zip(before, model.weights, model.partials, model.updates):
        want = L.orthogonalize(to_np(d), 5, E.QUINTIC, 1e-7, max(1.0, w0.shape[0] / w0.shape[1]) ** 0.5)
        g = to_np(u)
        # partials of a few tokens have singular values far below the largest, where fp16 products leave an error of some percent
        assert rms(g - want) <= 0.05 * rms(want)
        stepped = to_np(w0) - float(np.float32(0.5)) * g
        assert np.all(np.abs(to_np(w1) - stepped) <= 0.5 * bf16_ulp(stepped) + 1e-6)


def test_training_learns_and_decoding_continues_the_patterns():
    model, tokens, means = E.train(60)
    first, last = float(means[0]), float(means[-1])
    assert first < -3.5 and last > -0.35, (first, last)    # a uniform guess is -log 64 = -4.16; only each sequence's first tokens stay open
    said, logs = model.decode(tokens[:10], 20)
    assert torch.equal(said, tokens[10:30])
    assert bool((logs[..., 0] >= logs[..., 1]).all())
    B.relay_poll_status()


def test_a_step_can_be_captured_and_replayed():
    T, N, V, D = 40, 4, 64, 128
    model = E.RecurrentLM(V, D, T, N, seed=5)
    tokens = E.patterns(T + 1, N, V, 6)
    x, targets = model.one_hot(tokens[:-1]), tokens[1:].contiguous()
    d = torch.full((T, N), -1.0, device=DEV)
    top, ids = torch.empty(T, N, 3, device=DEV), torch.empty(T, N, 3, dtype=torch.int32, device=DEV)

    def step():
        model.forward(x, targets)
        B.relay_token_logprob(model.scores, targets, 1.0, model.logp, model.entropy, model.lse, top, ids)
        model.backward(x, targets, d)
        for p, u in zip(model.partials, model.updates):
            B.relay_orthogonalize(p, 5, E.QUINTIC, 1e-7, 1.0, u, model.ws)

    outs = [model.h, model.logp, model.entropy, model.lse, top, ids, model.dscores, model.dz, *model.partials, *model.updates]
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        step()
    for _ in range(2):
        for t in outs:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        B.relay_poll_status()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_small_shapes_pass_with_bounds_checks():
    r = child(["tests/test_gpu_recurrence.py", "tests/test_gpu_token_logprob.py", "tests/test_gpu_orthogonalize.py", "-k",
               "not offsets and not large and not long_and_wide and not many_rows and not alone and not refusals and not type_relation"])
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
