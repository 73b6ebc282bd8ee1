"""The operators of a state space language model at the ends of their types and lengths, and in forms that short sequences do not reach, against
the fp64 definitions.  Tolerances are those of the operators' own tests where nothing else is said."""
import numpy as np
import pytest
import torch

from oracle import state_space as S
from paper_1810_00952_b200 import binding as B

from parity import to_np, workspace

import test_gpu_causal_conv as C
import test_gpu_linear_logprob as H
import test_gpu_selective_scan as G
from test_gpu_bounds_check import child

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
LOWEST, INF = torch.finfo(torch.float32).min, float("inf")


def finite_where(got, want, what, rel=1e-4):
    """Finite, and close, where the definition is."""
    g, on = to_np(got), np.isfinite(want)
    assert on.any() and np.isfinite(g[on]).all(), (what, int((~np.isfinite(g[on])).sum()))
    assert np.abs(g[on] - want[on]).max() <= rel * np.abs(want[on]).max(), what


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


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 40, 130])
def test_without_a_skip_infinite_inputs_make_infinities(T):
    """A missing d is no term, not one of zero: 0 inf would be NaN."""
    t = G.make(T, 2, 20, 16, F32, seed=5, d=False, gated=True)
    for k in ("b", "c", "dy", "z"):
        t[k] = t[k].abs() + 0.1
    t["a"] /= 16
    t["u"][1, 0, 3] = INF
    y = _forward_y(t)[0]
    want, _ = S.selective_scan(*G.reference(t))
    assert np.isposinf(want[1:, 0, 3]).all() and np.array_equal(np.isposinf(to_np(y)), np.isposinf(want)) and not bool(torch.isnan(y).any())
    t["u"][1, 0, 3] = 1.0
    t["dy"][T - 1, 1, 7] = INF
    g = _gradient_raw(t, _forward_y(t)[2], {"du": (T, 2, 20)})
    assert bool(torch.isposinf(g["du"][:, 1, 7]).all())
    t["dy"][T - 1, 1, 7] = 1.0
    t["u"][1, 0, 3] = INF
    g = _gradient_raw(t, _forward_y(t)[2], {"dz": (T, 2, 20)})
    assert bool(torch.isposinf(g["dz"][1:, 0, 3]).all())


def _forward_y(t):
    """As G.forward, where results may be infinite or NaN."""
    T, Bn, D = t["u"].shape
    N = t["a"].shape[1]
    y, h, s = (torch.zeros(k, dtype=v, device=DEV) for k, v in (((T, Bn, D), t["u"].dtype), ((Bn, D, N), F32), ((-(-T // B.SCAN_SPAN), Bn, D, N), F32)))
    B.relay_selective_scan(*G.inputs(t), G.on(t["h0"]), G.on(t["lengths"]), t["softplus"], y, h, s)
    torch.cuda.synchronize()
    return y, h, s


def _gradient_raw(t, states, keep=None):
    T, Bn, D = t["u"].shape
    N, dt = t["a"].shape[1], t["u"].dtype
    shapes = dict(du=(T, Bn, D), ddelta=(T, Bn, D), da=(D, N), db=(T, Bn, N), dc=(T, Bn, N), dd=(D,), dz=(T, Bn, D), ddelta_bias=(D,), dh0=(Bn, D, N))
    gone = {"d" + k for k in ("d", "z", "delta_bias") if t[k] is None}
    o = {k: None if k in gone else torch.full(s, 3.0, dtype=dt if k in ("du", "ddelta", "db", "dc", "dz") else F32, device=DEV) for k, s in shapes.items()}
    ins = G.inputs(t)
    ws = workspace(B.relay_workspace_bytes_selective_scan_grad(ins[0], ins[2]), DEV).fill_(0xFF)
    B.relay_selective_scan_grad(*ins, G.on(t["lengths"]), t["softplus"], states, G.on(G.spoil(t, t["dy"])), G.on(t["dh_final"]), *o.values(), ws)
    torch.cuda.synchronize()
    return o


@pytest.mark.gpu
@pytest.mark.parametrize("N", [16, 10, 40])
@pytest.mark.parametrize("T", [33, 130])
def test_an_infinite_last_input_does_not_reach_behind_the_end(T, N):
    """The last input of a sequence is infinite: it makes infinities of what it enters, but the steps behind the end have no partials, and the
    partials of the decays, which it does not enter, are finite."""
    t = G.make(T, 6, 20, N, F32, seed=41, ragged=True, gated=False)
    t["lengths"][5] = T - 7
    t["u"][T - 8, 5, 3] = t["u"][T - 1, 0, 4] = t["u"][0, 2, 5] = INF
    y, h, s = _forward_y(t)
    with np.errstate(invalid="ignore"):
        want = S.selective_scan_grad(*G.reference(t), to_np(t["dy"]), to_np(t["dh_final"]))
    g = _gradient_raw(t, s)
    for i, end in enumerate(S._ends(t["lengths"].tolist(), T, 6)):
        for k in ("du", "ddelta", "db", "dc"):
            assert not bool(g[k][end:, i].any()), (k, i)
    for k in ("du", "ddelta", "da", "db", "dc", "dh0"):
        finite_where(g[k], want[k], k)


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


# ---- convolution -------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("D", [8, 9])
@pytest.mark.parametrize("K", [2, 4, 6])
def test_infinite_inputs_do_not_reach_the_filters_partials_from_behind_the_end(K, D):
    """dw[k] sums over the steps of the sequence alone: an infinite last input enters only under the last tap, and the inputs ahead of a sequence of
    no steps not at all."""
    t = C.make(40, 4, D, K, F32, F32, seed=K, ragged=False)
    t["lengths"] = torch.tensor([40, 21, 0, 33], dtype=torch.int32)
    t["x"][20, 1, 3] = t["x"][39, 0, 2] = INF
    t["before"][K - 2, 2, 5] = INF
    with np.errstate(invalid="ignore"):
        want = S.causal_conv_grad(to_np(t["x"]), to_np(t["w"]), to_np(t["b"]), to_np(t["before"]), t["lengths"].tolist(), False, to_np(t["dy"]), to_np(t["dafter"]))
    assert np.isfinite(want[1][:, 5]).all() and np.isfinite(want[1][:K - 1, 3]).all() and not np.isfinite(want[1][K - 1, 3])
    x, w = C.on(C.spoil(t, t["x"])), C.on(t["w"])
    dx, dw, db, dbefore = (torch.zeros(v, device=DEV) for v in ((40, 4, D), (K, D), (D,), (K - 1, 4, D)))
    ws = workspace(B.relay_workspace_bytes_causal_conv_grad(x, w), DEV).fill_(0xFF)
    B.relay_causal_conv_grad(x, w, C.on(t["b"]), C.on(t["before"]), C.on(t["lengths"]), B.ACT_NONE, C.on(C.spoil(t, t["dy"])), C.on(t["dafter"]), dx, dw, db, dbefore, ws)
    for got, v, what in ((dx, want[0], "dx"), (dw, want[1], "dw"), (db, want[2], "db"), (dbefore, want[3], "dbefore")):
        finite_where(got, v, what)


# ---- log-probabilities from the head's operands ----------------------------------------------------------------
def _log_terms(t, temperature):
    """Scores, lse and logp in 64 bits by torch."""
    x, w = t["x"].to(DEV).double(), (t["w"].T if t["tied"] else t["w"]).to(DEV).double()
    z = (x @ w) / temperature
    lse = torch.logsumexp(z, 1)
    return z, lse, z.gather(1, t["tokens"].to(DEV).long()[:, None])[:, 0] - lse


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("K", [1024, 4096, 65536])
def test_sums_that_fp32_holds_exactly_are_exact(K, tied):
    """One entry in a row of x, as in a table's row or a padded width, and weights in eighths: every score is an fp32 number and no sum rounds.  What
    is left, in units of 2^-24: of a score, the roundings of 1 / temperature, of log2(e) / temperature, of the maximum, of log(2), of its product
    and of the last sum, one each; of the sum of exponentials, made by an instruction good to 2^-22, 4 and as much again for its additions and log."""
    N, V = 65, 200
    r = np.random.default_rng(K)
    x, w = np.zeros((N, K)), r.integers(-16, 17, (K, V)) / 8
    x[np.arange(N), r.integers(0, K, N)] = r.integers(8, 32, N)
    t = dict(x=torch.from_numpy(x).to(BF16), w=torch.from_numpy(w.T.copy() if tied else w).to(BF16), tokens=torch.from_numpy(r.integers(0, V, N)).to(torch.int32),
             tied=tied)
    for temperature in (1.0, 0.75):
        logp, lse = H.forward(t, temperature)
        z, ws, wl = _log_terms(t, temperature)
        bound = (6 * z.abs().amax(1) + 16) * 2.0 ** -24
        assert bool(((lse.double() - ws).abs() <= bound).all()), float(((lse.double() - ws).abs() / bound).max())
        assert bool(((logp.double() - wl).abs() <= 2 * bound).all()), float(((logp.double() - wl).abs() / bound).max())


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("K", [512, 1024, 1032, 4096, 16384])
def test_long_contractions_lose_no_more_than_one_of_a_thousand_terms(K, tied):
    """Terms of one sign.  The tensor cores drop, at each addition of sixteen products, less than a unit in the last place (2^-23) of the sum so far,
    half of the final one on average: of 64 such additions, 64 x 2^-24 of the score.  Longer contractions are cut into pieces of 1024 whose sums
    are added with one rounding each.  The roundings behind the scores as above."""
    N, V = 40, 300
    r = np.random.default_rng(K)
    x, w = np.abs(r.normal(size=(N, K))), np.abs(r.normal(size=(K, V))) * 20 / (0.64 * K)
    t = dict(x=torch.from_numpy(x).to(BF16), w=torch.from_numpy(w.T.copy() if tied else w).to(BF16), tokens=torch.from_numpy(r.integers(0, V, N)).to(torch.int32),
             tied=tied, dlogp=torch.from_numpy(r.normal(size=N)).float())
    logp, lse = H.forward(t, 1.0)
    z, ws, wl = _log_terms(t, 1.0)
    bound = ((min(K, 1024) / 16 + K / 1024 + 6) * z.abs().amax(1) + 16) * 2.0 ** -24
    worst = float(((lse.double() - ws).abs() / bound).max())
    assert worst <= 1.0, worst
    H.check64(t, logp, lse, *H.gradient(t, 1.0, lse))


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
def test_rows_without_a_class_that_can_occur_have_no_part_in_the_gradient(tied):
    """lse = -inf, from x and from w: no partial passes, although the operands hold infinities."""
    N, K, V = 70, 24, 300
    t = H.make(N, K, V, BF16, seed=6, tied=tied, padded=False)
    flip = (lambda v: v.T) if tied else (lambda v: v)
    flip(t["w"])[0] = flip(t["w"])[0].abs() + 0.25
    _, clean = H.forward(t, 1.0)
    t["tokens"][::7] = -1
    none = torch.zeros(N, dtype=torch.bool)
    none[1::7] = True
    t["tokens"][none] = -1                                 # the same rows, without a token in place of without a class
    want = H.gradient(t, 1.0, clean)
    t["tokens"][none] = 5
    t["x"][none, 0] = -INF
    logp, lse = H.forward(t, 1.0)
    assert bool(torch.isneginf(lse.cpu()[none]).all()) and bool(torch.isneginf(logp.cpu()[none]).all()) and torch.equal(lse.cpu()[~none], clean.cpu()[~none])
    dx, dw = H.gradient(t, 1.0, lse)
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]) and not bool(dx.cpu()[none].any())
    # every class impossible, by w: no row has a part
    t["x"][:, 0] = t["x"][:, 0].abs().clamp(0.5, 4.0)
    flip(t["w"])[0] = -INF
    _, lse = H.forward(t, 1.0)
    assert bool(torch.isneginf(lse).all())
    dx, dw = H.gradient(t, 1.0, lse)
    assert not bool(dx.any()) and not bool(dw.any())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_rows_without_a_part_have_zero_partials_beside_infinite_weights(dt):
    t = H.make(70, 24, 300, dt, seed=6, padded=False)
    t["tokens"][::3] = -1
    t["w"][0, 100:] = -INF
    lse = torch.full((70,), 3.0, device=DEV)
    lse[1::3] = -INF
    gx, gw = torch.full((70, 24), 3.0, dtype=dt, device=DEV), torch.zeros(24, 300, dtype=dt, device=DEV)
    x, w = t["x"].to(DEV), t["w"].to(DEV)
    ws = workspace(B.relay_workspace_bytes_linear_logprob_grad(x, w, False), DEV)
    B.relay_linear_logprob_grad(x, w, False, t["tokens"].to(DEV), 1.0, lse, t["dlogp"].to(DEV), gx, gw, ws)
    assert not bool(gx[::3].any()) and not bool(gx[1::3].any())


@pytest.mark.gpu
def test_impossible_classes_in_the_gradient():
    """Weights of -inf beside finite ones: the partials of the scores are zero there, so that dw is what it is without these classes; dx is NaN where
    zero meets the infinite weight, and right in the other columns."""
    N, K, V = 64, 24, 200
    t = H.make(N, K, V, BF16, seed=8, padded=False)
    t["x"][:, 0] = t["x"][:, 0].abs().clamp(0.5, 4.0)
    t["tokens"] %= 150
    some = dict(t, w=t["w"][:, :150].contiguous())
    logp, lse = H.forward(some, 1.0)
    dx, dw = H.gradient(some, 1.0, lse)
    t["w"][0, 150:] = -INF
    l2, s2 = H.forward(t, 1.0)
    assert float((s2 - lse).abs().max()) <= 1e-5
    x, w = t["x"].to(DEV), t["w"].to(DEV)
    gx, gw = torch.empty_like(x), torch.empty_like(w)
    ws = workspace(B.relay_workspace_bytes_linear_logprob_grad(x, w, False), DEV)
    B.relay_linear_logprob_grad(x, w, False, t["tokens"].to(DEV), 1.0, lse, t["dlogp"].to(DEV), gx, gw, ws)
    assert torch.equal(gw[:, :150], dw) and not bool(gw[:, 150:].any())
    assert bool(torch.isnan(gx[:, 0]).all()) and torch.equal(gx[:, 1:], dx[:, 1:])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_calls_repeat_bit_for_bit(dt):
    """Sums in a fixed order: the same call gives the same bits, with products that are split too."""
    t = H.make(1500, 520, 5003, dt, seed=9, tied=dt == BF16)
    first = H.forward(t, 1.0)
    grads = H.gradient(t, 1.0, first[1])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(H.forward(t, 1.0), first))
        assert all(torch.equal(a, b) for a, b in zip(H.gradient(t, 1.0, first[1]), grads))


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("N", [1, 2, 3, 31, 33, 64, 100, 129, 300, 512])
def test_partials_of_few_rows_keep_sixteen_bits(N, tied):
    """A row's partials have one error in common where its token's own is rounded, and few rows do not average that out.  In two bf16 numbers a partial
    is off by half a step of the second, 2^-8 of at most 2^-8 of it, and by 512 2^-24 before (test_gpu_linear_logprob.py); the results are rounded
    once.  That counts fp32 sums as rounded to the nearest; the tensor cores' drop less than 2^-23 of the sum so far, of M at most, for every sixteen
    products: V / 16 2^-23 M in dx, which is 5e-4 M at 70,000 classes, and, of 2 N products, N / 8 2^-23 M in dw.  A partial rounded to bf16 alone is
    off by up to 3.9e-3 of itself.  Several pieces of the vocabulary from 100 rows on."""
    V = 70000 if N >= 100 else 1029
    K = 2056 if N >= 100 else 72
    t = H.make(N, K, V, BF16, seed=N, tied=tied, padded=N > 40)
    _, lse = H.forward(t, 0.7)
    dx, dw = H.gradient(t, 0.7, lse)
    x, w, dlogp, tokens = (t[k].to(DEV) for k in ("x", "w", "dlogp", "tokens"))
    x, w, dlogp, tokens = x.double(), (w.T if tied else w).double(), dlogp.double(), tokens.long()
    real = (tokens >= 0) & (tokens < V)
    z = (x @ w) / float(np.float32(0.7))
    slope = torch.where(real, dlogp, 0.0) / float(np.float32(0.7))
    dz = -slope[:, None] * torch.exp(z - torch.logsumexp(z, 1)[:, None])
    size = dz.abs()
    rows, at = torch.arange(N, device=DEV), tokens.clamp(0, V - 1)
    size[rows, at] += slope.abs()
    dz[rows, at] += slope
    flip = (lambda v: v.T) if tied else (lambda v: v)
    for got, want, m, terms in ((dx, dz @ w.T, size @ w.T.abs(), V), (dw, flip(x.T @ dz), flip(x.T.abs() @ size), 2 * N)):
        g, o = got.double(), want
        ulp = 2.0 ** (torch.floor(torch.log2(o.abs().clamp(min=2.0 ** -126))) - 7)
        bound = (512 * 2.0 ** -24 + 2.0 ** -16 + terms / 16 * 2.0 ** -23) * m + 0.5 * ulp * (1 + 2.0 ** -7) + 1e-37
        worst = float(((g - o).abs() / bound).max())
        assert worst <= 1.0, worst


@pytest.mark.gpu
def test_these_forms_pass_with_bounds_checks():
    r = child(["tests/test_gpu_state_space_ends.py", "-k", "not captured and not bounds_checks and not fp32_holds"])
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
