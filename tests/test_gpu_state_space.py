"""The operators of state space language models together, as examples/state_space_lm.py runs them: a training step whose groups are checked
against the definitions on the stored inputs, its gradients against differences, decoding, stream capture, calls that overlap on two
streams, and the bounds-check build."""
import os
import sys

import numpy as np
import pytest
import torch

from oracle import state_space as S
from paper_1810_00952_b200 import binding as B

from parity import bf16_ulp, to_np, workspace
from test_gpu_bounds_check import child
from test_gpu_linear_logprob import within as within_head
from test_gpu_selective_scan import within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

import state_space_lm as E  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def step(T=45, n=5, V=40, seed=3):
    model = E.StateSpaceLM(V, 32, 48, 16, T, n, seed=seed)
    tokens = E.patterns(T + 1, n, V, seed + 1)
    lengths = torch.tensor([T, 13, 1, 0, T - 1], dtype=torch.int32, device=DEV)
    x, targets = model.one_hot(tokens[:-1]), tokens[1:].clone()
    inside = torch.arange(T, device=DEV)[:, None] < lengths[None, :]
    targets[~inside] = -1                                  # padded positions name no token
    return model, x, targets, lengths, inside


def test_one_training_step_group_by_group():
    model, x, targets, lengths, inside = step()
    w = {k: to_np(v) for k, v in model.weights.items()}
    logp = model.forward(x, targets, lengths)
    model.backward(x, targets, torch.full_like(logp, -1.0), lengths)
    torch.cuda.synchronize()
    B.relay_poll_status()
    T, n, N = model.T, model.Bn, model.N
    ends = lengths.tolist()
    # convolution: eight products and the activation's roundings, 64 units of 2^-24 of the terms' sizes, then the store's half unit
    u, _ = S.causal_conv(to_np(model.x), w["w_conv"], w["b_conv"], None, ends, True)
    size, _ = S.causal_conv(np.abs(to_np(model.x)), np.abs(w["w_conv"]), None, None, ends, False)
    assert np.all(np.abs(to_np(model.u) - u) <= 64 * 2.0 ** -24 * 1.1 * size + 0.5 * bf16_ulp(u) * (1 + 2.0 ** -7))
    # scan
    bc = to_np(model.bc)
    args = [to_np(model.u), to_np(model.step), w["a"], bc[..., :N], bc[..., N:], w["skip"], to_np(model.z), w["b_step"], None, ends, True]
    within(model.y, S.selective_scan(*args)[0], S.selective_scan(*args, sizes=True)[0], 5 * T + 128, "y")
    assert not bool(model.y[~inside].any()) and not bool(model.u[~inside].any())
    # head
    h, flat = to_np(model.h).reshape(T * n, -1), to_np(targets).astype(int).reshape(-1)
    wl, ws = S.linear_logprob(h, w["table"].T, flat, 1.0)
    assert np.abs(to_np(logp).reshape(-1) - wl).max() <= 2e-5 * (1 + np.abs(ws).max() + np.abs(wl).max())
    dl = np.full(T * n, -1.0)
    dh, dt = S.linear_logprob_grad(h, w["table"].T, flat, 1.0, ws, dl)
    sh, st = S.linear_logprob_grad(h, w["table"].T, flat, 1.0, ws, dl, sizes=True)
    within_head(model.table1.T, dt, st, "table")
    # the scan's gradient on the stored partials of its result
    torch.cuda.synchronize()
    dy = torch.empty_like(model.y)
    B.relay_linear_logprob_grad(model.h, model.weights["table"], True, targets, 1.0, model.lse, torch.full_like(logp, -1.0), model.dh, None, model.ws)
    within_head(model.dh.view(T * n, -1), dh, sh, "dh")
    B.relay_fused_dense_act_grad(model.y, model.weights["w_out"], model.h, model.dh, B.ACT_NONE, dy, model.partials["w_out"], None, model.ws)
    g, size = S.selective_scan_grad(*args, to_np(dy), None), S.selective_scan_grad(*args, to_np(dy), None, sizes=True)
    for name, got in (("du", model.du), ("ddelta", model.dstep), ("dz", model.dz), ("da", model.partials["a"]), ("dd", model.partials["skip"]),
                      ("ddelta_bias", model.partials["b_step"])):
        within(got, g[name], size[name], 10 * T + 512, name)
    within(model.dbc, np.concatenate([g["db"], g["dc"]], 2), np.concatenate([size["db"], size["dc"]], 2), 10 * T + 512, "dbc")


def test_gradients_of_the_whole_model_match_differences():
    """Directional differences in the f32 weights, whose steps no rounding of weights disturbs.  The loss is a sum over T B log-probabilities;
    activations are stored in bf16, so every evaluation carries noise of some 2^-9 of a value in each of them, a fixed function of the weights
    that a wide difference averages over: where no weight moves by more than a twentieth of its size (or of one) the quotient follows the
    partials to a tenth."""
    model, x, targets, lengths, inside = step(T=40, n=5)
    logp = model.forward(x, targets, lengths)
    model.backward(x, targets, torch.full_like(logp, 1.0), lengths)
    partials = {k: v.clone() for k, v in model.partials.items()}
    g = torch.Generator(device=DEV).manual_seed(9)
    for name in ("w_conv", "a", "skip", "b_step", "b_conv"):
        w, d = model.weights[name], partials[name]
        v = d / d.norm() + 0.3 * torch.nn.functional.normalize(torch.randn(w.shape, generator=g, device=DEV).flatten(), dim=0).view(w.shape)
        h = 0.05 / float((v.abs() / w.abs().clamp(min=1.0)).max())
        keep, f = w.clone(), []
        for sign in (1.0, -1.0):
            w.copy_(keep + sign * h * v)
            f.append(float(model.forward(x, targets, lengths).double().sum()))
        w.copy_(keep)
        slope, want = (f[0] - f[1]) / (2 * h), float((d.double() * v.double()).sum())
        assert abs(slope - want) <= 0.1 * abs(want) + 1e-3, (name, slope, want)


def test_training_steps_and_decoding_run():
    model = E.StateSpaceLM(64, 32, 64, 16, 33, 4, seed=1)
    tokens = E.patterns(34, 4, 64, 2)
    for _ in range(3):
        logp = model.train_step(tokens, 0.1)
    assert bool(torch.isfinite(logp).all()) and all(bool(torch.isfinite(v).all()) and bool(v.any()) for v in model.partials.values())
    said, logs = model.decode(tokens[:8], 5)
    assert said.shape == (5, 4) and bool(((said >= 0) & (said < 64)).all()) and bool((logs[..., 0] >= logs[..., 1]).all())
    B.relay_poll_status()


def test_token_by_token_gives_the_sequence_s_scores():
    """What decoding computes for a prompt is what training computes for it: the same operators with T = 1 and their states."""
    model = E.StateSpaceLM(50, 32, 48, 16, 12, 3, seed=7)
    tokens = E.patterns(13, 3, 50, 8)
    model.forward(model.one_hot(tokens[:-1]), tokens[1:].clone())
    scores = torch.empty(3, 50, dtype=torch.bfloat16, device=DEV)
    B.relay_contract_act(model.h[-1].contiguous(), 0, model.weights["table"], 1, None, B.ACT_NONE, scores)
    ids, top = torch.empty(3, 4, dtype=torch.int32, device=DEV), torch.empty(3, 4, device=DEV)
    B.relay_token_logprob(scores, None, 1.0, None, None, None, top, ids)
    said, logs = model.decode(tokens[:12], 1)
    # the two differ by the order of fp32 sums, which the next bf16 rounding can turn into one unit of a value here and there
    assert float((logs[0] - top).abs().max()) <= 0.05
    B.relay_poll_status()


def test_a_step_can_be_captured_and_replayed():
    model, x, targets, lengths, _ = step(T=70, seed=5)
    d = torch.full((model.T, model.Bn), -1.0, device=DEV)
    names = ("u", "y", "states", "logp", "lse", "dh", "du", "dstep", "dbc", "dz", "dx")

    def run():
        model.forward(x, targets, lengths)
        model.backward(x, targets, d, lengths)

    outs = [getattr(model, k) for k in names] + list(model.partials.values())
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        run()
    for _ in range(2):
        for t in outs:
            t.fill_(7)
        g.replay()
        torch.cuda.synchronize()
        B.relay_poll_status()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))


def test_calls_overlap_on_two_streams():
    """Two training steps at once, each with its own buffers and workspace, on streams of their own: the results of each alone."""
    runs = []
    for seed in (11, 12):
        model, x, targets, lengths, _ = step(T=100, seed=seed)
        d = torch.full((model.T, model.Bn), -1.0, device=DEV)
        model.forward(x, targets, lengths)
        model.backward(x, targets, d, lengths)
        torch.cuda.synchronize()
        outs = [model.y, model.lse, model.du, model.dx] + list(model.partials.values())
        runs.append((model, x, targets, lengths, d, outs, [t.clone() for t in outs]))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for t in runs[0][5] + runs[1][5]:
        t.fill_(5)
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (model, x, targets, lengths, d, _, _) in zip(streams, runs):
            with torch.cuda.stream(s):
                model.forward(x, targets, lengths)
                model.backward(x, targets, d, lengths)
    torch.cuda.synchronize()
    B.relay_poll_status()
    for _, _, _, _, _, outs, want in runs:
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_results_do_not_depend_on_what_the_workspace_holds():
    model, x, targets, lengths, _ = step(T=50, seed=15)
    d = torch.full((model.T, model.Bn), -1.0, device=DEV)
    want = None
    for fill in (0, 0xFF, 0x7F):
        model.ws.fill_(fill)
        model.forward(x, targets, lengths)
        model.ws.fill_(fill)
        model.backward(x, targets, d, lengths)
        got = [t.clone() for t in (model.logp, model.du, model.dbc, model.dx, *model.partials.values())]
        assert want is None or all(torch.equal(a, b) for a, b in zip(want, got))
        want = got


def test_small_shapes_pass_with_bounds_checks():
    r = child(["tests/test_gpu_causal_conv.py", "tests/test_gpu_selective_scan.py", "tests/test_gpu_linear_logprob.py", "-k",
               "not offsets and not many_tiles and not pieces and not refusals and not type_relation"])
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
