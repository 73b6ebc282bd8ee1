"""The operators of a state space language model at the ends of their types and lengths, and in forms that short sequences do not reach, against
the fp64 definitions.  Tolerances are those of the operators' own tests where nothing else is said."""
import numpy as np
import pytest
import torch

from oracle import state_space as S
from paper_1810_00952_b200 import binding as B

from parity import to_np, workspace

import test_gpu_selective_scan as G

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
LOWEST, INF = torch.finfo(torch.float32).min, float("inf")


# ---- selective scan ----------------------------------------------------------------------------------------
def check(t):
    """As G.check.  The slope of the gate, q + z q (1 - q) with q the logistic function, is a sum whose terms cancel near z = -1.28, so what its
    rounding errors, and dz's, are measured against are its terms' absolute values as well."""
    T = t["u"].shape[0]
    y, h, s = G.forward(t)
    want, size = S.selective_scan(*G.reference(t), B.SCAN_SPAN), S.selective_scan(*G.reference(t), B.SCAN_SPAN, sizes=True)
    for k, got, w, m in zip(("y", "h_final", "states"), (y, h, s), want, size):
        G.within(got, w, m, 5 * T + 128, k)
    g = G.gradient(t, s)
    args = G.reference(t) + [to_np(t["dy"]), to_np(t["dh_final"])]
    want, size = S.selective_scan_grad(*args), S.selective_scan_grad(*args, sizes=True)
    z = to_np(t["z"])
    q = S._logistic(z)
    size["dz"] *= (q + np.abs(z) * q * (1 - q)) / np.abs(S._silu(z)[1])
    if t["packed"]:
        for v in (want, size):
            v["db"] = np.concatenate([v["db"], v["dc"]], axis=2)
    for k, v in g.items():
        G.within(v, want[k], size[k], 10 * T + 512, k)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T", [3, 33, 70, 130, 300])
def test_decays_that_leave_nothing(T, dt):
    """a of the type's lowest value, or so large that a log2(e) is beyond it: nothing is left of a state after any step, and what is added at the
    last one is the state, also where a chunk, or a block's whole part of the sequence, lies behind the end.  a = -inf is the same."""
    t = G.make(T, 6, 20, 16, dt, seed=21 + T, ragged=True, packed=True)
    t["a"][:4] = LOWEST
    t["a"][4:7, ::3] = -2.5e38
    check(t)
    want = G.forward(t)
    grads = G.gradient(t, want[2])
    t["a"][:4] = -INF
    assert all(torch.equal(a, b) for a, b in zip(G.forward(t), want))
    got = G.gradient(t, want[2])
    assert all(torch.equal(got[k], grads[k]) for k in grads)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T", [3, 33, 130])
def test_steps_of_no_length_keep_a_state_whatever_its_decay(T, dt):
    t = G.make(T, 6, 20, 16, dt, seed=31 + T, ragged=True)
    t["a"][:6] = LOWEST
    t["delta"][::2, :, :10] = -INF
    t["delta"][T - 1, 0] = -INF
    check(t)


def _forward_y(t):
    """As G.forward, where results may be infinite or NaN."""
    T, Bn, D = t["u"].shape
    N = t["a"].shape[1]
    y, h, s = (torch.zeros(k, dtype=v, device=DEV) for k, v in (((T, Bn, D), t["u"].dtype), ((Bn, D, N), F32), ((-(-T // B.SCAN_SPAN), Bn, D, N), F32)))
    B.relay_selective_scan(*G.inputs(t), G.on(t["h0"]), G.on(t["lengths"]), t["softplus"], y, h, s)
    torch.cuda.synchronize()
    return y, h, s


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("N", [17, 24, 32, 33, 64])
@pytest.mark.parametrize("T", [130, 300])
def test_shared_sequences_of_more_than_sixteen_states(T, N, dt):
    """Four blocks a sequence (130 steps) and eight (300), the last ones without a chunk, and sequences that end in an early block's part."""
    check(G.make(T, 2, 19, N, dt, seed=N + T, packed=True))
    t = G.make(T, 6, 20, N, dt, seed=N, ragged=True)
    t["lengths"][5] = 40
    check(t)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [16, 33])
def test_shared_sequences_keep_nan_in_its_channel_and_can_be_captured(N):
    T = 300
    t = G.make(T, 2, 20, N, F32, seed=10)
    clean, _, states = G.forward(t)
    grads = G.gradient(t, states)
    ins, h0, dy, dh = G.inputs(t), G.on(t["h0"]), G.on(t["dy"]), G.on(t["dh_final"])
    y, h, s = torch.empty_like(clean), torch.empty(2, 20, N, device=DEV), torch.empty_like(states)
    o = {k: torch.empty_like(v) for k, v in grads.items()}
    ws = workspace(B.relay_workspace_bytes_selective_scan_grad(ins[0], ins[2]), DEV)

    def run():
        B.relay_selective_scan(*ins, h0, None, True, y, h, s)
        B.relay_selective_scan_grad(*ins, None, True, s, dy, dh, *o.values(), ws)

    run()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        run()
    for _ in range(2):
        for v in (y, h, s, *o.values()):
            v.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        B.relay_poll_status()
        assert torch.equal(y, clean) and torch.equal(s, states) and all(torch.equal(o[k], grads[k]) for k in o)
    t["u"][T // 2, 1, 3] = float("nan")
    bad = torch.zeros(T, 2, 20, dtype=torch.bool)
    bad[T // 2:, 1, 3] = True
    y = _forward_y(t)[0].cpu()
    assert torch.equal(y[~bad], clean.cpu()[~bad]) and bool(torch.isnan(y[bad]).all())
