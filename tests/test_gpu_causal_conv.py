"""GPU parity: the short causal convolution and its gradient group against the fp64 definitions, through the C ABI.

Tolerances (parity.py): fp32 results 1e-4 relative with the floored denominator; bf16 results 1e-2 of the RMS plus half a unit in the
last place.  A sum of at most eight products of fp32 values is off by some 2^-22 of its terms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import state_space as S
from paper_1810_00952_b200 import binding as B

from parity import Guarded, assert_bf16, assert_f32, to_np, workspace

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make(T, Bn, D, K, dt, w_dt, seed, bias=True, before=True, ragged=False):
    r = np.random.default_rng(seed)
    rnd = lambda *s: torch.from_numpy(r.normal(size=s))
    t = dict(x=rnd(T, Bn, D).to(dt), w=rnd(K, D).to(w_dt), b=rnd(D).to(w_dt) if bias else None,
             before=rnd(K - 1, Bn, D).to(dt) if before else None, dy=rnd(T, Bn, D).to(dt), dafter=rnd(K - 1, Bn, D).to(dt), lengths=None)
    if ragged:
        n = r.integers(0, T + 1, Bn)
        n[:5] = [T, 0, min(1, T), T + 5, -3][:Bn]
        t["lengths"] = torch.from_numpy(n).to(torch.int32)
    return t


def spoil(t, x):
    """x with NaN in the steps behind the sequences' ends."""
    if t["lengths"] is None:
        return x
    x = x.clone()
    for i, n in enumerate(t["lengths"].tolist()):
        x[min(max(n, 0), x.shape[0]):, i] = float("nan")
    return x


def on(x):
    return None if x is None else x.to(DEV)


def forward(t, act, after=True):
    T, Bn, D = t["x"].shape
    K = t["w"].shape[0]
    y, last = Guarded((T, Bn, D), t["x"].dtype, DEV), Guarded((K - 1, Bn, D), t["x"].dtype, DEV)
    B.relay_causal_conv(on(spoil(t, t["x"])), on(t["w"]), on(t["b"]), on(t["before"]), on(t["lengths"]), act, y.t, last.t if after else None)
    torch.cuda.synchronize()
    return y.check(), last.check() if after else None


def gradient(t, act, dafter=True, dw=True, db=True, dbefore=True):
    T, Bn, D = t["x"].shape
    K = t["w"].shape[0]
    dt = t["x"].dtype
    o = dict(dx=Guarded((T, Bn, D), dt, DEV), dw=Guarded((K, D), F32, DEV), db=Guarded((D,), F32, DEV), dbefore=Guarded((K - 1, Bn, D), dt, DEV))
    x, w = on(spoil(t, t["x"])), on(t["w"])
    ws = workspace(B.relay_workspace_bytes_causal_conv_grad(x, w), DEV).fill_(0xFF)
    B.relay_causal_conv_grad(x, w, on(t["b"]), on(t["before"]), on(t["lengths"]), act, on(spoil(t, t["dy"])), on(t["dafter"]) if dafter else None,
                             o["dx"].t, o["dw"].t if dw else None, o["db"].t if db else None, o["dbefore"].t if dbefore else None, ws)
    torch.cuda.synchronize()
    wanted = dict(dx=True, dw=dw, db=db, dbefore=dbefore)
    return {k: v.check() for k, v in o.items() if wanted[k]}


def num(x):
    return None if x is None else to_np(x)


def check(t, act, dafter=True):
    silu = act == B.ACT_SILU
    args = (num(t["x"]), num(t["w"]), num(t["b"]), num(t["before"]), None if t["lengths"] is None else t["lengths"].tolist(), silu)
    same = assert_bf16 if t["x"].dtype == BF16 else assert_f32
    y, after = forward(t, act)
    wy, wafter = S.causal_conv(*args)
    same(y, wy, what="y")
    assert np.array_equal(to_np(after), wafter)
    g = gradient(t, act, dafter)
    wdx, wdw, wdb, wdbefore = S.causal_conv_grad(*args, num(t["dy"]), num(t["dafter"]) if dafter else None)
    same(g["dx"], wdx, what="dx"); same(g["dbefore"], wdbefore, what="dbefore")
    # a slope is off by a few 2^-22 (fp32), or with bf16 data by what the hardware's exponential leaves, 2^-21: sums of T B of them by less than
    # 1e-4 of their RMS
    assert_f32(g["dw"], wdw, what="dw"); assert_f32(g["db"], wdb, what="db")


SHAPES = [(1, 3, 16, 4), (2, 5, 8, 4), (7, 2, 24, 3), (37, 3, 10, 4), (130, 2, 33, 2), (65, 5, 40, 8), (20, 2, 7, 5), (9, 3, 12, 1),
          (300, 1, 264, 4), (1030, 2, 72, 4), (3, 1, 1, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_parity(shape, dt):
    T, Bn, D, K = shape
    check(make(T, Bn, D, K, dt, dt, seed=T + D), B.ACT_SILU)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", [(40, 6, 16, 4), (3, 5, 9, 4), (150, 7, 34, 3), (2, 5, 8, 8)])
def test_ragged_sequences_ignore_what_lies_behind_their_ends(shape, dt):
    T, Bn, D, K = shape
    check(make(T, Bn, D, K, dt, F32, seed=7, ragged=True), B.ACT_SILU)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_without_activation_bias_state_and_partial_of_the_state(dt):
    check(make(33, 2, 24, 4, dt, dt, seed=3, bias=False, before=False), B.ACT_NONE, dafter=False)


@pytest.mark.gpu
def test_optional_results_change_nothing_else():
    t = make(50, 3, 20, 4, BF16, F32, seed=4, ragged=True)
    y, _ = forward(t, B.ACT_SILU, after=False)
    assert torch.equal(y, forward(t, B.ACT_SILU)[0])
    full = gradient(t, B.ACT_SILU)
    for off in ("dw", "db", "dbefore"):
        part = gradient(t, B.ACT_SILU, **{off: False})
        assert off not in part and all(torch.equal(v, full[k]) for k, v in part.items())
    none = gradient(t, B.ACT_SILU, dw=False, db=False)
    assert torch.equal(none["dx"], full["dx"])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_token_by_token_is_the_whole_sequence(dt):
    """The state after a call is what the next one starts from; sums run in the same order, so the results are equal bit for bit."""
    t = make(11, 4, 16, 4, dt, dt, seed=5)
    whole, last = forward(t, B.ACT_SILU)
    state, y = on(t["before"]), torch.empty(1, 4, 16, dtype=dt, device=DEV)
    for k in range(11):
        after = torch.empty_like(state)
        B.relay_causal_conv(on(t["x"][k:k + 1]), on(t["w"]), on(t["b"]), state, None, B.ACT_SILU, y, after)
        assert torch.equal(y[0], whole[k])
        state = after
    assert torch.equal(state, last)


@pytest.mark.gpu
def test_no_steps_and_no_channels():
    t = make(0, 3, 8, 4, BF16, BF16, seed=6)
    _, after = forward(t, B.ACT_SILU)
    assert torch.equal(after.cpu(), t["before"])
    g = gradient(t, B.ACT_SILU)
    assert torch.equal(g["dbefore"].cpu(), t["dafter"]) and not g["dw"].any() and not g["db"].any()
    g = gradient(make(5, 0, 8, 4, F32, F32, seed=6), B.ACT_SILU)
    assert not g["dw"].any() and not g["db"].any()
    forward(make(5, 2, 0, 4, F32, F32, seed=6), B.ACT_SILU)


@pytest.mark.gpu
def test_infinities_and_nan_stay_in_their_channel_and_reach():
    t = make(40, 2, 16, 4, F32, F32, seed=8)
    clean, _ = forward(t, B.ACT_SILU)
    t["x"][10, 1, 3] = float("inf")
    t["x"][20, 0, 5] = float("nan")
    x = torch.empty(40, 2, 16, device=DEV)
    B.relay_causal_conv(on(t["x"]), on(t["w"]), on(t["b"]), on(t["before"]), None, B.ACT_SILU, x, None)
    touched = torch.zeros(40, 2, 16, dtype=torch.bool)
    touched[10:14, 1, 3] = True
    touched[20:24, 0, 5] = True
    assert torch.equal(x.cpu()[~touched], clean.cpu()[~touched])
    assert bool(torch.isnan(x.cpu()[20:24, 0, 5]).all())


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """2^31 and more elements: the last rows are those of a short call on the same rows."""
    T, Bn, D = 16400, 64, 2048
    x = torch.zeros(T, Bn, D, dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    tail = torch.randn(8, Bn, D, generator=g, device=DEV).to(BF16)
    x[-8:] = tail
    w, b = torch.randn(4, D, generator=g, device=DEV), torch.randn(D, generator=g, device=DEV)
    y, after = torch.empty_like(x), torch.empty(3, Bn, D, dtype=BF16, device=DEV)
    B.relay_causal_conv(x, w, b, None, None, B.ACT_SILU, y, after)
    short = torch.empty_like(tail)
    B.relay_causal_conv(tail, w, b, torch.zeros(3, Bn, D, dtype=BF16, device=DEV), None, B.ACT_SILU, short, None)
    assert torch.equal(y[-8:], short) and torch.equal(after, tail[-3:])
    B.relay_poll_status()


def test_type_relation():
    d = B.desc_of_type
    y, after = B.relay_infer_causal_conv(d(B.BF16, (5, 2, 8)), d(B.F32, (4, 8)))
    assert B._shape(y) == (5, 2, 8) and y.dtype == B.BF16 and B._shape(after) == (3, 2, 8) and after.dtype == B.BF16
    for x, w, status in ((d(B.I32, (5, 2, 8)), d(B.F32, (4, 8)), "ERR_DTYPE"), (d(B.BF16, (5, 8)), d(B.F32, (4, 8)), "ERR_RANK"),
                         (d(B.BF16, (5, 2, 8)), d(B.F32, (4, 9)), "ERR_SHAPE"), (d(B.BF16, (5, 2, 8)), d(B.F32, (9, 8)), "ERR_SHAPE"),
                         (d(B.BF16, (5, 2, 8)), d(B.F32, (0, 8)), "ERR_SHAPE"), (d(B.F32, (5, 2, 8)), d(B.BF16, (4, 8)), "ERR_DTYPE")):
        with pytest.raises(B.RelayError) as e:
            B.relay_infer_causal_conv(x, w)
        assert e.value.status_name == status


def test_refusals_leave_outputs_untouched(monkeypatch):
    """Everything here is refused on the host, before a launch; the tensors are host memory."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    z = lambda *s, dt=F32: torch.zeros(*s, dtype=dt)
    x, w, b, st, n = z(6, 2, 8), z(4, 8), z(8), z(3, 2, 8), z(2, dt=torch.int32)
    y, after, dw, db, dbf = (torch.full(s, 5.0) for s in ((6, 2, 8), (3, 2, 8), (4, 8), (8,), (3, 2, 8)))
    f, g, N = B.relay_causal_conv, B.relay_causal_conv_grad, B.ACT_NONE
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    cases = [(lambda: f(x, w, b, st, n, N, None, None), "ERR_NULL"),
             (lambda: f(x[0], w, b, st, n, N, y, None), "ERR_RANK"),
             (lambda: f(x, w[0], b, st, n, N, y, None), "ERR_RANK"),
             (lambda: f(x, w, b, st, n.long(), N, y, None), "ERR_DTYPE"),
             (lambda: f(x, w.bfloat16(), b, st, n, N, y, None), "ERR_DTYPE"),
             (lambda: f(x, w, b, st.bfloat16(), n, N, y, None), "ERR_DTYPE"),
             (lambda: f(x, w, b, st, n, N, y.bfloat16(), None), "ERR_DTYPE"),
             (lambda: f(x, z(9, 8), b, z(8, 2, 8), n, N, y, None), "ERR_SHAPE"),
             (lambda: f(x, w, z(7), st, n, N, y, None), "ERR_SHAPE"),
             (lambda: f(x, w, b, z(4, 2, 8), n, N, y, None), "ERR_SHAPE"),
             (lambda: f(x, w, b, st, z(3, dt=torch.int32), N, y, None), "ERR_SHAPE"),
             (lambda: f(x, w, b, st, n, B.ACT_RELU, y, None), "ERR_ATTR"),
             (lambda: f(x, w, b, st, n, 5, y, None), "ERR_ATTR"),
             (lambda: f(x, w, b, st, n, N, x, None), "ERR_ATTR"),
             (lambda: f(x, w, b, st, n, N, y, st), "ERR_ATTR"),
             (lambda: f(z(97)[1:].view(6, 2, 8), w, b, st, n, N, y, None), "ERR_ALIGN"),
             (lambda: g(x, w, b, st, n, N, None, None, y, dw, db, dbf, ws), "ERR_NULL"),
             (lambda: g(x, w, b, st, n, N, x, None, None, dw, db, dbf, ws), "ERR_NULL"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), st, y, dw.bfloat16(), db, dbf, ws), "ERR_DTYPE"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 9), st, y, dw, db, dbf, ws), "ERR_SHAPE"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), z(2, 2, 8), y, dw, db, dbf, ws), "ERR_SHAPE"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), st, y, dw, z(7), dbf, ws), "ERR_SHAPE"),
             (lambda: g(x, w, b, st, n, 2, z(6, 2, 8), st, y, dw, db, dbf, ws), "ERR_ATTR"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), st, y, dw, db, st, ws), "ERR_ATTR"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), st, y, dw, db, dbf, None), "ERR_WORKSPACE"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), st, y, dw, db, dbf, ws[:16]), "ERR_WORKSPACE"),
             (lambda: g(x, w, b, st, n, N, z(6, 2, 8), st, y, dw, db, dbf, ws[8:]), "ERR_WORKSPACE")]
    n0 = B.relay_launch_count()
    for i, (call, status) in enumerate(cases):
        with pytest.raises(B.RelayError) as e:
            call()
        assert e.value.status_name == status, (i, e.value)
    assert B.relay_launch_count() == n0
    assert all(bool((t == 5).all()) for t in (y, after, dw, db, dbf))
    with pytest.raises(ValueError):
        f(z(8, 2, 6).transpose(0, 2), w, b, st, n, N, y, None)
    assert B.relay_workspace_bytes_causal_conv_grad(x, z(4, 7)) == 0
