"""GPU parity: the gated linear recurrence and its gradient group against the fp64 definitions, through the C ABI.

Tolerances (parity.py): fp32 results 1e-4 relative with the floored denominator; bf16 results 1e-2 of the RMS plus half a
unit in the last place.  The state is fp32 in both; a coefficient's relative error of a few 2^-23 moves a sum over a span of
S steps by at most S times that, 1e-5 at the spans of some tens of steps that these gates give."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import language as L
from paper_1810_00952_b200 import binding as B

from parity import Guarded, assert_bf16, assert_f32, bf16_ulp, to_np

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
GATES = [B.GATE_GIVEN, B.GATE_SIGMOID, B.GATE_MIX]


def make(T, Bn, D, dt, gate, packed, ragged, seed, h0=True):
    r = np.random.default_rng(seed)
    f = r.uniform(0.3, 0.99, (T, Bn, D)) if gate == B.GATE_GIVEN else r.normal(1.5, 2.0, (T, Bn, D))
    t = dict(f=torch.from_numpy(f).to(dt), u=torch.from_numpy(r.normal(size=(T, Bn, D))).to(dt),
             h0=torch.from_numpy(r.normal(size=(Bn, D))).float() if h0 else None,
             dh_all=torch.from_numpy(r.normal(size=(T, Bn, D))), dh_final=torch.from_numpy(r.normal(size=(Bn, D))).float(), lengths=None)
    if ragged:
        n = r.integers(0, T + 1, Bn)
        n[:4] = [T, 0, min(1, T), T + 5][:Bn]
        t["lengths"] = torch.from_numpy(n).to(torch.int32)
    t["packed"] = torch.cat([t["f"], t["u"]], dim=2).contiguous() if packed else None
    return t


def spoil(t, x, value):
    """x with `value` in the steps behind the sequences' ends."""
    if t["lengths"] is not None:
        x = x.clone()
        for b, n in enumerate(t["lengths"].tolist()):
            x[min(max(n, 0), x.shape[0]):, b] = value
    return x


def on(x):
    return None if x is None else x.to(DEV)


def run_forward(t, gate, out_dt, stream=None, final=True):
    f, u = (t["packed"], None) if t["packed"] is not None else (t["f"], t["u"])
    T, Bn, D = t["f"].shape
    h, last = Guarded((T, Bn, D), out_dt, DEV), Guarded((Bn, D), F32, DEV)
    f, u = on(spoil(t, f, float("nan"))), on(None if u is None else spoil(t, u, float("nan")))
    B.relay_gated_recurrence(f, u, on(t["h0"]), on(t["lengths"]), gate, h.t, last.t if final else None)
    torch.cuda.synchronize()
    return h.check(), last.check() if final else None


def run_grad(t, gate, h_all, dh0=True, dh_final=True):
    f, u = (t["packed"], None) if t["packed"] is not None else (t["f"], t["u"])
    T, Bn, D = t["f"].shape
    nan = float("nan")
    df, d0 = Guarded(tuple(f.shape), f.dtype, DEV), Guarded((Bn, D), F32, DEV)
    du = None if u is None else Guarded((T, Bn, D), f.dtype, DEV)
    dh = spoil(t, t["dh_all"].to(h_all.dtype), nan)
    B.relay_gated_recurrence_grad(on(spoil(t, f, nan)), on(None if u is None else spoil(t, u, nan)), on(t["h0"]), on(t["lengths"]), gate,
                                  h_all, on(dh), on(t["dh_final"]) if dh_final else None, df.t, None if du is None else du.t,
                                  d0.t if dh0 else None)
    torch.cuda.synchronize()
    df = df.check()
    if u is None:
        df, du = df[..., :D], df[..., D:]
    else:
        du = du.check()
    return df, du, d0.check() if dh0 else None


def expect(t, gate):
    T, Bn, D = t["f"].shape
    f, u = to_np(t["f"]), to_np(t["u"])
    h0 = to_np(t["h0"]) if t["h0"] is not None else np.zeros((Bn, D))
    return f, u, h0, None if t["lengths"] is None else t["lengths"].tolist()


def check_case(T, Bn, D, dt, gate, packed, ragged, out_dt=None, seed=0, h0=True):
    t = make(T, Bn, D, dt, gate, packed, ragged, seed + T * 7 + D, h0)
    out_dt = out_dt or dt
    f, u, h0v, n = expect(t, gate)
    want, want_last = L.gated_recurrence(f, u, h0v, n, gate)
    h, last = run_forward(t, gate, out_dt)
    (assert_bf16 if out_dt == BF16 else assert_f32)(h, want, what="h_all")
    assert_f32(last, want_last, what="h_final")
    # the gradient group is given the stored h_all
    df, du, d0 = run_grad(t, gate, h)
    want_df, want_du, want_d0 = L.gated_recurrence_grad(f, u, h0v, n, gate, to_np(h), to_np(t["dh_all"].to(out_dt)), to_np(t["dh_final"]))
    check = assert_bf16 if dt == BF16 else assert_f32
    check(df, want_df, what="df"); check(du, want_du, what="du")
    assert_f32(d0, want_d0, what="dh0")


# one step, spans of the sequence around every power of two that a split could use, odd and even channel counts
@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 12, 13, 15, 16, 17, 33, 127, 128, 129, 300, 1025])
@pytest.mark.parametrize("Bn,D", [(1, 1), (3, 64), (2, 67), (5, 130)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_lengths_of_the_sequence(T, Bn, D, dt):
    check_case(T, Bn, D, dt, B.GATE_MIX, packed=T % 2 == 0, ragged=False)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("dt,out_dt", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("D", [96, 33])
def test_gates_layouts_and_types(gate, packed, ragged, dt, out_dt, D):
    check_case(150, 6, D, dt, gate, packed, ragged, out_dt)


@pytest.mark.gpu
@pytest.mark.parametrize("T,Bn,D", [(4100, 1, 64), (4100, 2, 6), (2500, 1, 515), (700, 40, 100), (40, 9, 2000)])
@pytest.mark.parametrize("ragged", [False, True])
def test_long_and_wide(T, Bn, D, ragged):
    check_case(T, Bn, D, BF16, B.GATE_SIGMOID, True, ragged)
    check_case(T, Bn, D, F32, B.GATE_MIX, False, ragged, seed=5)


# rows of an even width that are not whole 16-byte pieces, with enough channels for two a lane: either side of every rule
@pytest.mark.gpu
@pytest.mark.parametrize("T", [33, 64, 65, 200])
@pytest.mark.parametrize("Bn,D", [(2, 1022), (1, 66), (7, 170)])
@pytest.mark.parametrize("dt,out_dt", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("gate,packed,ragged", [(B.GATE_GIVEN, True, False), (B.GATE_SIGMOID, False, True), (B.GATE_MIX, True, True)])
def test_even_rows_that_are_not_whole_pieces(T, Bn, D, dt, out_dt, gate, packed, ragged):
    check_case(T, Bn, D, dt, gate, packed, ragged, out_dt)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 40, 700])
def test_absent_states_are_zero(T):
    check_case(T, 3, 66, F32, B.GATE_MIX, False, False, h0=False)
    t = make(T, 3, 66, BF16, B.GATE_SIGMOID, True, False, 9)
    h, _ = run_forward(t, B.GATE_SIGMOID, BF16, final=False)
    a = run_grad(t, B.GATE_SIGMOID, h, dh_final=False)
    b = run_grad(dict(t, dh_final=torch.zeros(3, 66)), B.GATE_SIGMOID, h, dh0=False)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and b[2] is None


@pytest.mark.gpu
@pytest.mark.parametrize("T", [3, 600])
def test_gates_at_their_ends(T):
    """sigmoid arguments of +-100 and the infinities: coefficients of exactly one and zero, and no NaN."""
    t = make(T, 2, 8, F32, B.GATE_MIX, False, False, 3)
    t["f"][:, 0] = torch.tensor([100.0, -100.0, float("inf"), float("-inf"), 30.0, -30.0, 0.0, 88.0])
    for gate in (B.GATE_SIGMOID, B.GATE_MIX):
        f, u, h0, n = expect(t, gate)
        h, last = run_forward(t, gate, F32)
        want, want_last = L.gated_recurrence(f, u, h0, n, gate)
        assert_f32(h, want, what="h_all"); assert_f32(last, want_last, what="h_final")
        df, du, d0 = run_grad(t, gate, h)
        for got, w in zip((df, du, d0), L.gated_recurrence_grad(f, u, h0, n, gate, to_np(h), to_np(t["dh_all"].float()), to_np(t["dh_final"]))):
            assert_f32(got, w)


@pytest.mark.gpu
@pytest.mark.parametrize("T,D", [(9, 64), (9, 33), (40, 64), (40, 33), (40, 34), (300, 64), (300, 33)])
@pytest.mark.parametrize("dt,out_dt", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("gate", [B.GATE_SIGMOID, B.GATE_MIX])
def test_shut_gates_keep_their_relative_precision(T, D, dt, out_dt, gate):
    """One step whose gates are shut (f from -8 to -30) among open ones, values of zero and partials of one sign, so that no sum
    cancels: states and partials there are products with the small coefficient.  Relative error: of the exponential and its argument
    at most 4e-6, of the reciprocal and the products 1e-6, of the sums over the open steps (a = 0.95, some 20 of them) 3e-6; the bound is
    2e-5, and half a unit in the last place where the result is bf16."""
    t = make(T, 2, D, dt, gate, False, False, 41)
    at = T // 2
    t["lengths"] = torch.full((2,), T, dtype=torch.int32)                 # rows of D channels, not of 2 D
    t["f"][:] = 3.0
    t["f"][at] = torch.linspace(-8.0, -30.0, D).to(dt)
    t["u"][:] = 0.0
    if gate == B.GATE_MIX:
        t["u"][at - 1] = 1.0                                              # a state that has not decayed
    else:
        t["u"][at - 1] = 2.0
    t["dh_all"], t["dh_final"] = t["dh_all"].abs() + 0.1, t["dh_final"].abs()
    t["h0"] = t["h0"].abs() + 0.1
    f, u, h0, n = expect(t, gate)

    def near(got, want, what):
        g = to_np(got)
        slack = 0.5 * bf16_ulp(want) if got.dtype == BF16 else 0.0
        assert np.all(np.abs(g - want) <= 2e-5 * np.abs(want) + slack), (what, np.max(np.abs(g - want) / np.maximum(np.abs(want), 1e-300)))

    h, _ = run_forward(t, gate, out_dt)
    near(h[at], L.gated_recurrence(f, u, h0, n, gate)[0][at], "h")
    df, du, d0 = run_grad(t, gate, h)
    want = L.gated_recurrence_grad(f, u, h0, n, gate, to_np(h), to_np(t["dh_all"].to(out_dt)), to_np(t["dh_final"]))
    near(df[at], want[0][at], "df"); near(du[at], want[1][at], "du")
    # one step alone: what reaches the initial state is a g and nothing else
    t1 = {k: v[at:at + 1].contiguous() if k in ("f", "u", "dh_all") else v for k, v in t.items()}
    t1["lengths"] = None
    h, _ = run_forward(t1, gate, out_dt)
    near(run_grad(t1, gate, h)[2], L.gated_recurrence_grad(f[at:at + 1], u[at:at + 1], h0, None, gate, to_np(h), to_np(t1["dh_all"].to(out_dt)),
                                                         to_np(t["dh_final"]))[2], "dh0")


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 14, 90, 700])
@pytest.mark.parametrize("Bn,D", [(2, 72), (3, 33)])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("gate", GATES)
def test_nan_stays_in_its_channel_and_after_its_step(T, Bn, D, dt, gate):
    t = make(T, Bn, D, dt, gate, False, False, 31)

    def forward(t):
        h, last = torch.zeros(T, Bn, D, dtype=dt, device=DEV), torch.zeros(Bn, D, device=DEV)
        B.relay_gated_recurrence(on(t["f"]), on(t["u"]), on(t["h0"]), None, gate, h, last)
        return h.cpu(), last.cpu()

    clean = forward(t)[0]
    at = T // 2
    for name, channel in (("f", 3), ("u", 17)):
        v = t[name].clone()
        v[at, 1, channel] = float("nan")
        h, last = forward(dict(t, **{name: v}))
        bad = torch.zeros(T, Bn, D, dtype=torch.bool)
        bad[at:, 1, channel] = True
        assert torch.equal(torch.isnan(h), bad) and torch.equal(torch.isnan(last), bad[-1])
        assert torch.equal(h[~bad], clean[~bad])


@pytest.mark.gpu
def test_long_memory_keeps_its_precision():
    """Gates at 1 - 2^-10 over 5000 steps: the running mean of a constant is that constant, and of ones from zero it is 1 - a^t."""
    T = 5000
    f = torch.full((T, 1, 66), float(np.log(1023.0)))
    t = dict(f=f, u=torch.ones(T, 1, 66), h0=None, lengths=None, packed=None, dh_all=torch.zeros(T, 1, 66), dh_final=torch.zeros(1, 66))
    h, _ = run_forward(t, B.GATE_MIX, F32)
    fv = float(f[0, 0, 0])
    a = 1 / (1 + np.exp(-np.float64(fv)))
    want = 1 - a ** np.arange(1, T + 1)
    assert_f32(h, np.broadcast_to(want[:, None, None], (T, 1, 66)))
    # one coefficient is off by a few units of 2^-24 (relative in 1 - a); 2e-6 leaves room for four of them and the sum's own
    assert np.max(np.abs(to_np(h)[-1] / want[-1] - 1)) < 2e-6


@pytest.mark.gpu
@pytest.mark.parametrize("T", [50, 900])
def test_gradient_against_differences_of_the_forward_call(T):
    """Directional differences: the forward call is linear in u and h0, so a step of any size is exact up to rounding; f is
    probed by a small one, whose error is of its square."""
    t = make(T, 3, 34, F32, B.GATE_MIX, False, True, 11)
    r = np.random.default_rng(12)
    spoiled = spoil(t, t["dh_all"], 0.0)

    def scalar(**kw):
        h, last = run_forward(dict(t, **kw), B.GATE_MIX, F32)
        return float((to_np(h) * to_np(spoiled)).sum() + (to_np(last) * to_np(t["dh_final"])).sum())

    h, _ = run_forward(t, B.GATE_MIX, F32)
    df, du, d0 = run_grad(dict(t, dh_all=spoiled), B.GATE_MIX, h)
    for name, got, eps, tol in (("u", du, 1.0, 2e-5), ("h0", d0, 1.0, 2e-5), ("f", df, 1e-2, 2e-4)):
        v = torch.from_numpy(r.normal(size=tuple(t[name].shape))).float()
        fd = (scalar(**{name: t[name] + eps * v}) - scalar(**{name: t[name] - eps * v})) / (2 * eps)
        an = float((to_np(got) * to_np(v)).sum())
        scale = float(np.sqrt((to_np(got) ** 2).sum()))
        assert abs(fd - an) <= tol * max(scale, abs(an)), (name, fd, an)


@pytest.mark.gpu
def test_same_bits_every_time_and_on_another_stream():
    t = make(1500, 2, 300, BF16, B.GATE_MIX, True, False, 21)
    h, last = run_forward(t, B.GATE_MIX, BF16)
    g = run_grad(t, B.GATE_MIX, h)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            h2, last2 = run_forward(t, B.GATE_MIX, BF16)
            assert torch.equal(h, h2) and torch.equal(last, last2)
            assert all(torch.equal(a, b) for a, b in zip(g, run_grad(t, B.GATE_MIX, h2)))


@pytest.mark.gpu
def test_step_by_step_decoding_continues_a_sequence():
    t = make(600, 4, 128, BF16, B.GATE_MIX, True, False, 31)
    h, _ = run_forward(t, B.GATE_MIX, F32)
    x = on(t["packed"])
    state, nxt = on(t["h0"]).clone(), torch.empty(4, 128, device=DEV)
    _, state = run_forward(dict(t, f=t["f"][:500], u=t["u"][:500], packed=t["packed"][:500].contiguous()), B.GATE_MIX, F32)
    for k in range(500, 600):
        out = torch.empty(1, 4, 128, device=DEV)
        B.relay_gated_recurrence(x[k:k + 1], None, state, None, B.GATE_MIX, out, nxt)
        state, nxt = nxt, state
        assert_f32(out[0], to_np(h[k]))


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """2^31 + elements a tensor: with a = 0 the state is the value itself, with a = 1 and one value per channel it stays."""
    T, C = 33000, 65536
    f = torch.zeros(T, 1, C, dtype=BF16, device=DEV)
    u = torch.arange(T * 8, device=DEV, dtype=torch.int32).remainder_(251).to(BF16).repeat(C // 8).view(T, 1, C)
    h = torch.full((T, 1, C), float("nan"), dtype=BF16, device=DEV)
    B.relay_gated_recurrence(f, u, None, None, B.GATE_GIVEN, h, None)
    assert torch.equal(h, u)
    df, du = torch.empty_like(f), torch.empty_like(f)
    B.relay_gated_recurrence_grad(f, u, None, None, B.GATE_GIVEN, h, u, None, df, du, None)
    assert torch.equal(du, u)
    assert torch.equal(df[1:], (u[1:].float() * u[:-1].float()).to(BF16)) and not bool(df[0].any())


@pytest.mark.gpu
def test_empty_sizes():
    for shape in [(0, 2, 8), (4, 0, 8), (4, 2, 0)]:
        x = torch.zeros(shape, device=DEV)
        h0 = torch.full(shape[1:], 3.0, device=DEV)
        last, d0 = torch.zeros(shape[1:], device=DEV), torch.zeros(shape[1:], device=DEV)
        B.relay_gated_recurrence(x, x.clone(), h0, None, B.GATE_MIX, torch.empty(shape, device=DEV), last)
        assert torch.equal(last, h0)
        B.relay_gated_recurrence_grad(x, x.clone(), h0, None, B.GATE_MIX, x.clone(), x.clone(), h0, torch.empty(shape, device=DEV),
                                      torch.empty(shape, device=DEV), d0)
        assert torch.equal(d0, h0)
    torch.cuda.synchronize()


def test_type_relation():
    d = B.desc_of_type
    h, last = B.relay_infer_gated_recurrence(d(B.BF16, (7, 2, 10)), d(B.BF16, (7, 2, 10)))
    assert (h.dtype, list(h.shape[:3]), last.dtype, list(last.shape[:2])) == (B.BF16, [7, 2, 10], B.F32, [2, 10])
    h, last = B.relay_infer_gated_recurrence(d(B.F32, (7, 2, 10)))
    assert (h.dtype, list(h.shape[:3])) == (B.F32, [7, 2, 5])


def test_refusals_leave_outputs_untouched(monkeypatch):
    """Everything here is refused on the host, before a launch; the tensors are host memory."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    f, u = torch.zeros(4, 2, 8), torch.zeros(4, 2, 8)
    h, s, n = torch.full((4, 2, 8), 5.0), torch.full((2, 8), 5.0), torch.zeros(2, dtype=torch.int32)
    z = lambda *shape, dt=F32: torch.zeros(*shape, dtype=dt)
    fwd = B.relay_gated_recurrence
    cases = [(lambda: fwd(f, None, None, None, 0, None, None), "ERR_NULL"),
             (lambda: fwd(f[0], u, None, None, 0, h, None), "ERR_RANK"),
             (lambda: fwd(f, u, z(2, 8, 1), None, 0, h, None), "ERR_RANK"),
             (lambda: fwd(z(4, 2, 8, dt=torch.int32), None, None, None, 0, h, None), "ERR_DTYPE"),
             (lambda: fwd(f, u.bfloat16(), None, None, 0, h, None), "ERR_DTYPE"),
             (lambda: fwd(f, u, None, None, 0, h.bfloat16(), None), "ERR_DTYPE"),
             (lambda: fwd(f, u, z(2, 8, dt=BF16), None, 0, h, None), "ERR_DTYPE"),
             (lambda: fwd(f, u, None, n.long(), 0, h, None), "ERR_DTYPE"),
             (lambda: fwd(f, z(4, 2, 7), None, None, 0, h, None), "ERR_SHAPE"),
             (lambda: fwd(z(4, 2, 7), None, None, None, 0, h, None), "ERR_SHAPE"),         # two blocks of an odd axis
             (lambda: fwd(f, None, None, None, 0, h, None), "ERR_SHAPE"),                  # packed: D = 4
             (lambda: fwd(f, u, z(3, 8), None, 0, h, None), "ERR_SHAPE"),
             (lambda: fwd(f, u, None, z(3, dt=torch.int32), 0, h, None), "ERR_SHAPE"),
             (lambda: fwd(f, u, None, None, 3, h, None), "ERR_ATTR"),
             (lambda: fwd(f, u, None, None, 0, f, None), "ERR_ATTR"),                      # output over an input
             (lambda: fwd(f, u, s, None, 0, h, s), "ERR_ATTR"),
             (lambda: fwd(z(65)[1:].view(4, 2, 8), u, None, None, 0, h, None), "ERR_ALIGN")]
    g, h2 = B.relay_gated_recurrence_grad, z(4, 2, 8)
    df, du = torch.full((4, 2, 8), 5.0), torch.full((4, 2, 8), 5.0)
    cases += [(lambda: g(f, u, None, None, 0, h, None, None, df, du, None), "ERR_NULL"),
              (lambda: g(f, u, None, None, 0, h, h2, None, df, None, None), "ERR_NULL"),
              (lambda: g(f, u, None, None, 0, h, h2.bfloat16(), None, df, du, None), "ERR_DTYPE"),
              (lambda: g(f, u, None, None, 0, h, h2, None, df.bfloat16(), du, None), "ERR_DTYPE"),
              (lambda: g(f, u, None, None, 0, h, h2, None, z(4, 2, 16), du, None), "ERR_SHAPE"),
              (lambda: g(f, u, None, None, 0, h, h2, z(2, 9), df, du, None), "ERR_SHAPE"),
              (lambda: g(f, u, None, None, 0, h, h2, None, df, df, None), "ERR_ATTR"),
              (lambda: g(f, u, None, None, 0, h, h2, s, df, du, s), "ERR_ATTR"),
              (lambda: g(z(4, 2, 16), None, None, None, 0, h, h2, None, z(4, 2, 16), du, None), "ERR_ATTR")]
    n0 = B.relay_launch_count()
    for i, (call, status) in enumerate(cases):
        with pytest.raises(B.RelayError) as e:
            call()
        assert e.value.status_name == status, (i, e.value)
    assert B.relay_launch_count() == n0
    for t in (h, s, df, du):
        assert bool((t == 5.0).all())
