"""GPU parity: the selective scan and its gradient group against the fp64 definitions, through the C ABI.

Tolerances.  Results are sums of terms that may cancel, so errors are measured against the sums of the terms' absolute values, M.  With eps =
2^-24: a term delta u b is made with 12 eps (softplus 8, two products, one conversion); in each step that it lives through it is multiplied by a
decay that is off by 2.4 eps (the hardware's exponential) and 12 eps of its exponent, and rounded with one more, and once again where spans are
joined.  The exponents of all steps together are X where the term has shrunk to exp(-X) of itself, and X exp(-X) < 0.4, so after T steps a term
is off by less than (5 T + 20) eps.  The product with c, the sum over N <= 64 states and d u add N at most, the gate 16 eps: (5 T + 128) eps M.  The
gradient's terms are products of two such chains: (10 T + 256) eps M, and the sums over T B steps and D channels, added up in groups of at most
32 and 64, fewer than 256 more.  bf16 results are rounded once more, by half a unit in the last place."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import state_space as S
from paper_1810_00952_b200 import binding as B

from parity import Guarded, assert_bf16, assert_f32, bf16_ulp, to_np, workspace

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
SEQ = ("u", "delta", "b", "c", "z")


def make(T, Bn, D, N, dt, seed, gated=True, softplus=True, packed=False, ragged=False, d=True, bias=True, h0=True):
    r = np.random.default_rng(seed)
    rnd = lambda *s: torch.from_numpy(r.normal(size=s))
    steps = np.exp(r.uniform(np.log(1e-3), np.log(0.5), (T, Bn, D)))
    t = dict(u=rnd(T, Bn, D).to(dt), delta=(torch.from_numpy(np.log(np.expm1(steps))) if softplus else torch.from_numpy(steps)).to(dt),
             a=-torch.from_numpy(r.uniform(0.1, N, (D, N))).float(), b=rnd(T, Bn, N).to(dt), c=rnd(T, Bn, N).to(dt),
             d=rnd(D).float() if d else None, z=rnd(T, Bn, D).to(dt) if gated else None,
             delta_bias=(0.1 * rnd(D)).float() if bias else None, h0=rnd(Bn, D, N).float() if h0 else None,
             dy=rnd(T, Bn, D).to(dt), dh_final=rnd(Bn, D, N).float(), lengths=None, softplus=softplus, packed=packed)
    if bias and not softplus:
        t["delta_bias"] = t["delta_bias"].abs()
    if ragged:
        n = r.integers(0, T + 1, Bn)
        n[:5] = [T, 0, min(1, T), T + 5, -3][:Bn]
        t["lengths"] = torch.from_numpy(n).to(torch.int32)
    return t


def spoil(t, x):
    if t["lengths"] is None or x is None:
        return x
    x = x.clone()
    for i, n in enumerate(t["lengths"].tolist()):
        x[min(max(n, 0), x.shape[0]):, i] = float("nan")
    return x


def on(x):
    return None if x is None else x.to(DEV)


def inputs(t):
    q = {k: on(spoil(t, t[k]) if k in SEQ else t[k]) for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias")}
    if t["packed"]:
        q["b"], q["c"] = torch.cat([q["b"], q["c"]], dim=2).contiguous(), None
    return list(q.values())


def forward(t, states=True, final=True):
    T, Bn, D = t["u"].shape
    N = t["a"].shape[1]
    y, h, s = Guarded((T, Bn, D), t["u"].dtype, DEV), Guarded((Bn, D, N), F32, DEV), Guarded((-(-T // B.SCAN_SPAN), Bn, D, N), F32, DEV)
    B.relay_selective_scan(*inputs(t), on(t["h0"]), on(t["lengths"]), t["softplus"], y.t, h.t if final else None, s.t if states else None)
    torch.cuda.synchronize()
    return y.check(), h.check() if final else None, s.check() if states else None


def gradient(t, states, dh_final=True, off=()):
    T, Bn, D = t["u"].shape
    N, dt = t["a"].shape[1], t["u"].dtype
    shapes = dict(du=(T, Bn, D), ddelta=(T, Bn, D), da=(D, N), db=(T, Bn, 2 * N if t["packed"] else N), dc=(T, Bn, N), dd=(D,), dz=(T, Bn, D),
                  ddelta_bias=(D,), dh0=(Bn, D, N))
    gone = set(off) | ({"dc"} if t["packed"] else set()) | {"d" + k for k in ("d", "z", "delta_bias") if t[k] is None}
    o = {k: None if k in gone else Guarded(s, dt if k in ("du", "ddelta", "db", "dc", "dz") else F32, DEV) for k, s in shapes.items()}
    ins = inputs(t)
    ws = workspace(B.relay_workspace_bytes_selective_scan_grad(ins[0], ins[2]), DEV).fill_(0xFF)
    B.relay_selective_scan_grad(*ins, on(t["lengths"]), t["softplus"], states, on(spoil(t, t["dy"])), on(t["dh_final"]) if dh_final else None,
                                *[None if v is None else v.t for v in o.values()], ws)
    torch.cuda.synchronize()
    return {k: v.check() for k, v in o.items() if v is not None}


def num(x):
    return None if x is None else to_np(x)


def reference(t):
    return [num(t[k]) for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias", "h0")] + [None if t["lengths"] is None else t["lengths"].tolist(),
                                                                                               t["softplus"]]


def within(got, want, size, units, what):
    g = to_np(got)
    assert g.shape == want.shape and np.all(np.isfinite(g)), what
    bound = units * 2.0 ** -24 * size + (0.5 * bf16_ulp(want) * (1 + 2.0 ** -7) if got.dtype == BF16 else 0.0) + 1e-37
    worst = (np.abs(g - want) / bound).max() if g.size else 0.0
    assert worst <= 1.0, (what, float(worst))


def check(t, dh_final=True):
    T = t["u"].shape[0]
    y, h, s = forward(t)
    want, size = S.selective_scan(*reference(t), B.SCAN_SPAN), S.selective_scan(*reference(t), B.SCAN_SPAN, sizes=True)
    for k, got, w, m in zip(("y", "h_final", "states"), (y, h, s), want, size):
        within(got, w, m, 5 * T + 128, k)
    g = gradient(t, s, dh_final)
    args = reference(t) + [num(t["dy"]), num(t["dh_final"]) if dh_final else None]
    want, size = S.selective_scan_grad(*args), S.selective_scan_grad(*args, sizes=True)
    if t["packed"]:
        for q in (want, size):
            q["db"] = np.concatenate([q["db"], q["dc"]], axis=2)
    for k, v in g.items():
        within(v, want[k], size[k], 10 * T + 512, k)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", [(1, 3, 16, 16), (2, 2, 5, 3), (4, 1, 33, 16), (5, 2, 17, 16), (8, 2, 16, 7), (31, 1, 20, 16), (32, 2, 34, 16),
                                   (33, 2, 32, 16), (100, 3, 48, 16), (257, 1, 18, 12), (70, 2, 9, 1)])
def test_parity(shape, dt):
    T, Bn, D, N = shape
    check(make(T, Bn, D, N, dt, seed=T + N, packed=T % 2 == 0))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("N", [17, 24, 32, 33, 48, 64])
def test_more_than_sixteen_states(N, dt):
    check(make(67, 2, 19, N, dt, seed=N, packed=True))
    check(make(3, 2, 19, N, dt, seed=N + 1))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", [(3, 6, 8, 16), (40, 6, 18, 16), (130, 7, 33, 16), (75, 6, 20, 40)])
def test_ragged_sequences_ignore_what_lies_behind_their_ends(shape, dt):
    T, Bn, D, N = shape
    check(make(T, Bn, D, N, dt, seed=7, ragged=True, packed=D % 2 == 0))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("gated,softplus,d,bias,h0", [(False, True, True, True, True), (True, False, True, True, True), (True, True, False, False, True),
                                                      (False, False, False, False, False)])
def test_optional_operands(gated, softplus, d, bias, h0, dt):
    for T in (3, 45):
        check(make(T, 2, 24, 16, dt, seed=T, gated=gated, softplus=softplus, d=d, bias=bias, h0=h0), dh_final=h0)


@pytest.mark.gpu
def test_optional_results_change_nothing_else():
    t = make(50, 3, 20, 16, BF16, seed=4, ragged=True)
    y, h, s = forward(t)
    for states, final in ((False, True), (True, False), (False, False)):
        y2, h2, s2 = forward(t, states, final)
        assert torch.equal(y, y2) and (h2 is None or torch.equal(h, h2)) and (s2 is None or torch.equal(s, s2))
    full = gradient(t, s)
    for off in ("dd", "ddelta_bias", "dh0"):
        assert all(torch.equal(v, full[k]) for k, v in gradient(t, s, off=(off,)).items())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_token_by_token_is_the_whole_sequence(dt):
    t = make(70, 3, 24, 16, dt, seed=5)
    y, h, _ = forward(t)
    state, row = on(t["h0"]), torch.empty(1, 3, 24, dtype=dt, device=DEV)
    rows = []
    for k in range(70):
        q = [v[k:k + 1] if n in SEQ else v for n, v in zip(("u", "delta", "a", "b", "c", "d", "z", "delta_bias"), inputs(t))]
        after = torch.empty_like(state)
        B.relay_selective_scan(*q, state, None, True, row, after, None)
        rows.append(row.clone())
        state = after
    (assert_bf16 if dt == BF16 else assert_f32)(torch.cat(rows), to_np(y))
    assert_f32(state, to_np(h))


@pytest.mark.gpu
def test_states_saved_by_pieces_are_those_of_the_whole():
    """A sequence handed over in calls of whole spans leaves the same states behind."""
    t = make(96, 2, 16, 16, F32, seed=6)
    _, h, s = forward(t)
    ins, state, parts = inputs(t), on(t["h0"]), []
    for k in (0, 32):
        e = 32 if k == 0 else 96
        q = [v[k:e].contiguous() if n in SEQ else v for n, v in zip(("u", "delta", "a", "b", "c", "d", "z", "delta_bias"), ins)]
        y, after, st = torch.empty_like(q[0]), torch.empty_like(state), torch.empty((e - k) // 32, 2, 16, 16, device=DEV)
        B.relay_selective_scan(*q, state, None, True, y, after, st)
        parts.append(st)
        state = after
    assert_f32(torch.cat(parts), to_np(s)); assert_f32(state, to_np(h))


@pytest.mark.gpu
def test_no_steps_and_no_channels():
    t = make(0, 2, 8, 16, BF16, seed=8)
    _, h, s = forward(t)
    assert torch.equal(h.cpu(), t["h0"])
    g = gradient(t, s)
    assert torch.equal(g["dh0"].cpu(), t["dh_final"]) and not g["da"].any() and not g["dd"].any() and not g["ddelta_bias"].any()
    t = make(9, 0, 8, 16, F32, seed=8)
    g = gradient(t, forward(t)[2])
    assert not g["da"].any() and not g["dd"].any() and not g["ddelta_bias"].any()
    t = make(9, 2, 0, 16, F32, seed=8)
    forward(t)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_steep_decays_and_long_steps(dt):
    """Decays that underflow to zero, steps that leave a state untouched, and softplus far out on both sides."""
    t = make(80, 2, 16, 16, dt, seed=9, bias=False)
    t["a"][:4] = -3.0e4
    t["a"][4:8] = 0.0
    t["delta"][::3] = 40.0
    t["delta"][1::3] = -40.0
    check(t)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T", [3, 80, 300])
def test_steps_of_no_length(T, dt):
    """delta of -inf or of the type's lowest value: softplus is zero there, the state stays, and no partial passes through."""
    t = make(T, 2, 20, 16, dt, seed=12)
    t["delta"][::2, :, :10] = float("-inf")
    t["delta"][1::3, :, 5:] = torch.finfo(dt).min
    t["delta"][T - 1, 0] = float("-inf")
    check(t)


@pytest.mark.gpu
def test_nan_stays_in_its_channel_and_behind_its_step():
    for T in (4, 80):
        t = make(T, 2, 20, 16, F32, seed=10)
        clean, _, _ = forward(t)
        t["u"][T // 2, 1, 3] = float("nan")
        y = torch.empty(T, 2, 20, device=DEV)
        B.relay_selective_scan(*inputs(t), on(t["h0"]), None, True, y, None, None)
        bad = torch.zeros(T, 2, 20, dtype=torch.bool)
        bad[T // 2:, 1, 3] = True
        assert torch.equal(y.cpu()[~bad], clean.cpu()[~bad]) and bool(torch.isnan(y.cpu()[bad]).all())


@pytest.mark.gpu
def test_large_offsets():
    """2^31 and more elements of a sequence: the last steps are those of a short call from the state before them."""
    T, Bn, D, N = 4200, 64, 8192, 16
    u = torch.zeros(T, Bn, D, dtype=BF16, device=DEV)
    bc = torch.zeros(T, Bn, 2 * N, dtype=BF16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    u[-8:] = torch.randn(8, Bn, D, generator=g, device=DEV).to(BF16)
    bc[-8:] = torch.randn(8, Bn, 2 * N, generator=g, device=DEV).to(BF16)
    a = -torch.rand(D, N, generator=g, device=DEV)
    y, h = torch.empty_like(u), torch.empty(Bn, D, N, device=DEV)
    B.relay_selective_scan(u, u, a, bc, None, None, None, None, None, None, True, y, h, None)
    y2, h2 = torch.empty_like(u[-8:]), torch.empty_like(h)
    B.relay_selective_scan(u[-8:], u[-8:], a, bc[-8:], None, None, None, None, None, None, True, y2, h2, None)
    B.relay_poll_status()
    assert not bool(y[:-8].any())
    assert float((y[-8:].float() - y2.float()).abs().max()) <= 2.0 ** -7 * float(y2.float().abs().max())
    assert float((h - h2).abs().max()) <= 1e-5 * float(h2.abs().max())


def test_type_relation():
    d = B.desc_of_type
    y, h, s = B.relay_infer_selective_scan(d(B.BF16, (65, 2, 8)), d(B.F32, (8, 16)))
    assert B._shape(y) == (65, 2, 8) and y.dtype == B.BF16 and B._shape(h) == (2, 8, 16) and h.dtype == B.F32
    assert B._shape(s) == (3, 2, 8, 16) and s.dtype == B.F32 and B.SCAN_SPAN == 32
    for u, a, status in ((d(B.I32, (5, 2, 8)), d(B.F32, (8, 16)), "ERR_DTYPE"), (d(B.BF16, (5, 8)), d(B.F32, (8, 16)), "ERR_RANK"),
                         (d(B.BF16, (5, 2, 8)), d(B.BF16, (8, 16)), "ERR_DTYPE"), (d(B.BF16, (5, 2, 8)), d(B.F32, (9, 16)), "ERR_SHAPE"),
                         (d(B.BF16, (5, 2, 8)), d(B.F32, (8, 65)), "ERR_SHAPE"), (d(B.BF16, (5, 2, 8)), d(B.F32, (8, 0)), "ERR_SHAPE")):
        with pytest.raises(B.RelayError) as e:
            B.relay_infer_selective_scan(u, a)
        assert e.value.status_name == status


def test_refusals_leave_outputs_untouched(monkeypatch):
    """Everything here is refused on the host, before a launch; the tensors are host memory."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    z = lambda *s, dt=F32: torch.zeros(*s, dtype=dt)
    good = dict(u=z(40, 2, 8), delta=z(40, 2, 8), a=z(8, 16), b=z(40, 2, 16), c=z(40, 2, 16), d=z(8), z=z(40, 2, 8), delta_bias=z(8),
                h0=z(2, 8, 16), lengths=z(2, dt=torch.int32), softplus=1, y=torch.full((40, 2, 8), 5.0), h_final=torch.full((2, 8, 16), 5.0),
                states=torch.full((2, 2, 8, 16), 5.0))
    five = lambda *s: torch.full(s, 5.0)
    grad = {k: good[k] for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias", "lengths", "softplus")}
    grad.update(states=z(2, 2, 8, 16), dy=z(40, 2, 8), dh_final=z(2, 8, 16), du=five(40, 2, 8), ddelta=five(40, 2, 8), da=five(8, 16), db=five(40, 2, 16),
                dc=five(40, 2, 16), dd=five(8), dz=five(40, 2, 8), ddelta_bias=five(8), dh0=five(2, 8, 16), ws=torch.zeros(1 << 20, dtype=torch.uint8))
    lib = B.lib()

    def call(fn, base, **changes):
        q = dict(base, **changes)
        if fn is B.relay_selective_scan and not isinstance(q["softplus"], bool) and q["softplus"] not in (0, 1):   # past the binding's bool()
            B._check(lib.relay_selective_scan(*[B._packed(q[k]) for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias", "h0", "lengths")],
                                              q["softplus"], B._packed(q["y"]), None, None, None))
        fn(*q.values())

    f, g = B.relay_selective_scan, B.relay_selective_scan_grad
    cases = [(f, good, dict(u=None), "ERR_NULL"), (f, good, dict(delta=None), "ERR_NULL"), (f, good, dict(a=None), "ERR_NULL"),
             (f, good, dict(b=None), "ERR_NULL"), (f, good, dict(y=None), "ERR_NULL"),
             (f, good, dict(u=z(40, 8)), "ERR_RANK"), (f, good, dict(h0=z(2, 8)), "ERR_RANK"), (f, good, dict(states=z(2, 8, 16)), "ERR_RANK"),
             (f, good, dict(delta=z(40, 2, 8, dt=BF16)), "ERR_DTYPE"), (f, good, dict(a=z(8, 16, dt=BF16)), "ERR_DTYPE"),
             (f, good, dict(d=z(8, dt=BF16)), "ERR_DTYPE"), (f, good, dict(lengths=z(2, dt=torch.int64)), "ERR_DTYPE"),
             (f, good, dict(y=z(40, 2, 8, dt=BF16)), "ERR_DTYPE"),
             (f, good, dict(a=z(8, 65)), "ERR_SHAPE"), (f, good, dict(b=z(40, 2, 15)), "ERR_SHAPE"), (f, good, dict(c=None), "ERR_SHAPE"),
             (f, good, dict(z=z(40, 2, 9)), "ERR_SHAPE"), (f, good, dict(delta_bias=z(9)), "ERR_SHAPE"), (f, good, dict(h_final=z(2, 8, 15)), "ERR_SHAPE"),
             (f, good, dict(states=z(1, 2, 8, 16)), "ERR_SHAPE"), (f, good, dict(lengths=z(3, dt=torch.int32)), "ERR_SHAPE"),
             (f, good, dict(softplus=2), "ERR_ATTR"), (f, good, dict(y=good["u"]), "ERR_ATTR"), (f, good, dict(h_final=good["h0"]), "ERR_ATTR"),
             (f, good, dict(z=z(641)[1:].view(40, 2, 8)), "ERR_ALIGN"),
             (g, grad, dict(states=None), "ERR_NULL"), (g, grad, dict(dy=None), "ERR_NULL"), (g, grad, dict(da=None), "ERR_NULL"),
             (g, grad, dict(dc=None), "ERR_NULL"), (g, grad, dict(dz=None), "ERR_NULL"),
             (g, grad, dict(dd=z(8, dt=BF16)), "ERR_DTYPE"), (g, grad, dict(du=z(40, 2, 8, dt=BF16)), "ERR_DTYPE"),
             (g, grad, dict(states=z(3, 2, 8, 16)), "ERR_SHAPE"), (g, grad, dict(dh0=z(2, 8, 15)), "ERR_SHAPE"),
             (g, grad, dict(z=None), "ERR_ATTR"), (g, grad, dict(d=None), "ERR_ATTR"), (g, grad, dict(delta_bias=None), "ERR_ATTR"),
             (g, grad, dict(c=None, b=z(40, 2, 32), db=z(40, 2, 32)), "ERR_ATTR"), (g, grad, dict(du=grad["ddelta"]), "ERR_ATTR"),
             (g, grad, dict(ws=None), "ERR_WORKSPACE"), (g, grad, dict(ws=grad["ws"][:64]), "ERR_WORKSPACE"), (g, grad, dict(ws=grad["ws"][8:]), "ERR_WORKSPACE")]
    n0 = B.relay_launch_count()
    for i, (fn, base, changes, status) in enumerate(cases):
        with pytest.raises(B.RelayError) as e:
            call(fn, base, **changes)
        assert e.value.status_name == status, (i, e.value)
    assert B.relay_launch_count() == n0
    kept = [good[k] for k in ("y", "h_final", "states")] + [grad[k] for k in ("du", "ddelta", "da", "db", "dc", "dd", "dz", "ddelta_bias", "dh0")]
    assert all(bool((t == 5).all()) for t in kept)
    assert B.relay_workspace_bytes_selective_scan_grad(good["u"], z(9, 16)) == 0
