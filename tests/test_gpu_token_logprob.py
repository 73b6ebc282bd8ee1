"""GPU parity: log-probabilities of given tokens, entropies, top alternatives and their gradient group against the fp64
definitions, through the C ABI.

Tolerances (parity.py): 1e-4 with the floored denominator for fp32 results (an exponential is good to some 1e-6 at scores of a few
tens), 1e-2 of the RMS plus half a unit in the last place for bf16 gradients.  Ids are compared exactly."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import language as L
from paper_1810_00952_b200 import binding as B

from parity import Guarded, assert_bf16, assert_f32, to_np

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


def scores(N, V, dt, seed, masked=0.0):
    r = np.random.default_rng(seed)
    z = r.normal(0, 3, (N, V))
    if masked:
        z[r.random((N, V)) < masked] = -np.inf
    tok = r.integers(0, V, N)
    tok[::5] = -1
    if N > 3:
        tok[3] = V
    return torch.from_numpy(z).to(dt), torch.from_numpy(tok).to(torch.int32), r


def stored(temperature):
    """The value that crosses the C ABI as a float."""
    return float(np.float32(temperature))


def forward(z, tok, temperature=1.0, top=0):
    lead = tuple(z.shape[:-1])
    o = dict(logp=Guarded(lead, F32, DEV), entropy=Guarded(lead, F32, DEV), lse=Guarded(lead, F32, DEV))
    if top:
        o["top_logp"], o["top_ids"] = Guarded((*lead, top), F32, DEV), Guarded((*lead, top), torch.int32, DEV)
    B.relay_token_logprob(z.to(DEV), tok.to(DEV), temperature, o["logp"].t, o["entropy"].t, o["lse"].t, o["top_logp"].t if top else None,
                          o["top_ids"].t if top else None)
    torch.cuda.synchronize()
    return {k: v.check(all_written=False) for k, v in o.items()}


def same(got, want, what=""):
    """assert_f32 where the definition is finite; the very same infinities and NaN elsewhere."""
    g, w = to_np(got), np.asarray(want, dtype=np.float64)
    fine = np.isfinite(w)
    np.testing.assert_array_equal(g[~fine], w[~fine], err_msg=what)
    if fine.any():
        assert_f32(torch.from_numpy(g[fine]), w[fine], what=what)


def check_forward(z, tok, temperature=1.0, top=0):
    o = forward(z, tok, temperature, top)
    w = L.token_logprob(to_np(z), tok.numpy(), stored(temperature), top)
    for k in ("logp", "entropy", "lse"):
        same(o[k], w[k], k)
    if top:
        np.testing.assert_array_equal(o["top_ids"].cpu().numpy(), w["top_ids"])
        same(o["top_logp"], w["top_logp"], "top_logp")
    return o, w


def check_grad(z, tok, temperature, o, r, with_entropy=True):
    N = z.shape[0]
    dlogp = torch.from_numpy(r.normal(size=N)).float()
    dent = torch.from_numpy(r.normal(size=N)).float() if with_entropy else None
    dz = Guarded(tuple(z.shape), z.dtype, DEV)
    B.relay_token_logprob_grad(z.to(DEV), tok.to(DEV), temperature, o["lse"], o["entropy"] if with_entropy else None, dlogp.to(DEV),
                               dent.to(DEV) if with_entropy else None, dz.t)
    torch.cuda.synchronize()
    want = L.token_logprob_grad(to_np(z), tok.numpy(), stored(temperature), to_np(o["lse"]), to_np(o["entropy"]), to_np(dlogp),
                                to_np(dent) if with_entropy else None)
    (assert_f32 if z.dtype == F32 else assert_bf16)(dz.check(), want, what="dscores")


# a row shorter than a vector, than a warp, than a block; odd rows (every alignment of the start); rows of several blocks
SIZES = [(1, 1), (3, 2), (5, 7), (17, 33), (9, 255), (4, 1000), (13, 1027), (3, 4096), (6, 5003), (2, 32768), (3, 50021), (1, 131072), (1, 262147)]


@pytest.mark.gpu
@pytest.mark.parametrize("N,V", SIZES)
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_rows_of_all_sizes(N, V, dt, temperature):
    z, tok, r = scores(N, V, dt, N * 1009 + V)
    o, _ = check_forward(z, tok, temperature, top=min(V, 20))
    check_grad(z, tok, temperature, o, r)
    check_grad(z, tok, temperature, o, r, with_entropy=False)


@pytest.mark.gpu
@pytest.mark.parametrize("N", [2, 20, 150, 700, 3000])
@pytest.mark.parametrize("V", [40, 2050, 9000])
def test_many_rows(N, V):
    z, tok, r = scores(N, V, BF16, N + V)
    some = slice(0, N, max(1, N // 40))
    o = forward(z, tok, 1.0, 5)
    w = L.token_logprob(to_np(z[some]), tok[some].numpy(), 1.0, 5)
    for k in ("logp", "entropy", "lse", "top_logp"):
        same(o[k][some], w[k], k)
    np.testing.assert_array_equal(o["top_ids"][some].cpu().numpy(), w["top_ids"])
    assert torch.allclose(o["lse"].cpu(), torch.logsumexp(z.float(), 1), rtol=1e-5, atol=1e-5)


@pytest.mark.gpu
@pytest.mark.parametrize("N,V", [(5, 100), (5, 9001), (2, 60000), (320, 2000), (320, 601)])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("top", [20, 21, 24, 25, 31, 32, 33, 63, 64])
def test_numbers_of_alternatives_around_the_changes_of_their_bound(N, V, dt, top):
    r = np.random.default_rng(V + top)
    z = torch.from_numpy(r.normal(0, 3, (N, V))).to(dt)
    z[0] = torch.arange(V).to(dt)                        # rising; in bf16 with many equal ones
    z[1, : V - 3] = -INF                                 # fewer than asked for can occur
    some = [0, 1, N // 2, N - 1]
    o = forward(z, torch.zeros(N, dtype=torch.int32), 1.0, top)
    w = L.token_logprob(to_np(z[some]), np.zeros(len(some), int), 1.0, top)
    np.testing.assert_array_equal(o["top_ids"][some].cpu().numpy(), w["top_ids"])
    same(o["top_logp"][some], w["top_logp"], "top_logp")


@pytest.mark.gpu
@pytest.mark.parametrize("V", [11, 300, 5003, 40000])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("top", [1, 8, 64])
def test_ties_go_to_the_lower_id(V, dt, top):
    top = min(top, V)
    r = np.random.default_rng(V)
    z = torch.from_numpy(r.integers(-2, 3, (6, V)).astype(np.float64)).to(dt)
    z[1] = 4.0                                           # all equal
    z[2] = torch.arange(V).to(dt)                        # rising: the largest come last
    z[3] = -torch.arange(V).to(dt)
    z[4] = -INF; z[4, V // 2] = 0.0                      # one class that can occur
    z[5, ::2] = 0.0; z[5, 1::2] = -0.0                   # signed zeros are equal
    check_forward(z, torch.zeros(6, dtype=torch.int32), 1.0, top)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [5, 1000, 33001])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_masked_rows_infinities_and_nan(V, dt):
    z, tok, r = scores(9, V, dt, V, masked=0.5)
    tok[:] = V - 1
    low = torch.finfo(dt).min
    z[0] = -INF                                          # the mask leaves nothing
    z[1] = low                                           # masks of the type's lowest value: all equal, a uniform row
    z[2] = low; z[2, 1] = 5.0
    z[3, 2] = NAN
    z[4, V - 1] = INF
    z[5] = -INF; z[5, V - 1] = -3.0                      # certainty
    z[6] = -INF; z[6, 0] = 1.0                           # the token cannot occur
    z[7, 0] = NAN; z[7, V - 1] = NAN
    z[8] = 1.0e4 * torch.arange(V).remainder(3).to(dt)   # far apart, no overflow
    o, _ = check_forward(z, tok, 1.0, min(V, 6))
    fine = [0, 1, 2, 5, 6, 8]
    check_grad(z[fine], tok[fine], 1.0, {k: o[k][fine].contiguous() for k in ("lse", "entropy")}, r)
    check_grad(z[fine], tok[fine], 1.0, {k: o[k][fine].contiguous() for k in ("lse", "entropy")}, r, with_entropy=False)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [2, 7, 1000, 33001, 200000])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("temperature", [1.0, 0.6])
def test_large_maxima_beside_masked_classes(V, dt, temperature):
    """The distance from a large maximum to a masked class is not a finite number: such a class adds nothing to the entropy."""
    low = torch.finfo(dt).min
    z = torch.empty(8, V, dtype=dt)
    for row, (m, rest) in enumerate([(1e32, -INF), (1e32, low), (3e37, -INF), (3e37, low), (1e30, low), (1e29, -INF), (-1e32, -INF), (-1e37, low)]):
        z[row] = rest
        z[row, V // 2] = m
        z[row, ::97] = m                                   # several equal ones: the entropy is the logarithm of their number
    z[7, -1] = low
    tok = torch.full((8,), V // 2, dtype=torch.int32)
    o, w = forward(z, tok, temperature, 1), L.token_logprob(to_np(z), tok.numpy(), stored(temperature), 1)
    np.testing.assert_array_equal(o["top_ids"].cpu().numpy(), w["top_ids"])
    with np.errstate(over="ignore"):
        for k in ("logp", "entropy", "lse", "top_logp"):
            same(o[k], w[k].astype(np.float32), k)         # as stored: what is below the type's range is -inf


@pytest.mark.gpu
@pytest.mark.parametrize("V", [3, 1000, 33001])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("temperature,weight", [(1e-10, 1.0), (1e-5, 1e20), (1.0, 1e25)])
def test_gradient_of_impossible_classes_under_steep_slopes(V, dt, temperature, weight):
    """dentropy / temperature of 1e10 to 1e25 times a log-probability far below any exponential's range: the partials there are zero.
    The other classes' scores differ by no more than the temperature, so that they have probabilities.  Their term lp + H cancels to
    rounding where they are all equal, so one of them stands apart; the tolerance is the parity tests' own."""
    low = torch.finfo(dt).min
    z = torch.zeros(4, V, dtype=dt)
    z[:, 0] = temperature                                  # one class e times as probable
    z[:, -1] = torch.tensor([-INF, low, -1e20, -1e4])
    tok = torch.zeros(4, dtype=torch.int32)
    o = forward(z, tok, temperature)
    dlogp, dent = torch.full((4,), weight), torch.full((4,), weight)
    dz = Guarded((4, V), dt, DEV)
    B.relay_token_logprob_grad(z.to(DEV), tok.to(DEV), temperature, o["lse"], o["entropy"], dlogp.to(DEV), dent.to(DEV), dz.t)
    torch.cuda.synchronize()
    got = dz.check()
    assert not bool(got[:, -1].any())
    want = L.token_logprob_grad(to_np(z), tok.numpy(), stored(temperature), to_np(o["lse"]), to_np(o["entropy"]), to_np(dlogp), to_np(dent))
    (assert_f32 if dt == F32 else assert_bf16)(got, want, what="dscores")


@pytest.mark.gpu
@pytest.mark.parametrize("V", [5, 1000, 33001])
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("temperature", [1e-45, 2e-38, 1e-20, 9e19, 1e21, 1e30, 1e38, 3e38])
def test_temperatures_at_the_ends_of_their_range(V, dt, temperature):
    """Scores at the temperature's own scale beside masks of -inf and of the lowest value: at 1e38 the lowest value is no mask, and
    -inf still is."""
    t = max(stored(temperature), float(np.finfo(np.float32).tiny))
    r = np.random.default_rng(V)
    x = np.clip(2 * t * r.normal(size=(7, V)), -3e38, 3e38)
    masked = r.random(V) < 0.5
    masked[0] = False
    x[1, masked] = -np.inf
    z = torch.from_numpy(x).to(dt)
    low = torch.finfo(dt).min
    z[2, torch.from_numpy(masked)] = low
    z[3] = 0.0; z[3, -1] = -INF
    z[4] = low
    z[5] = -INF; z[5, 0] = 0.0
    if t >= 1e30:
        z[6, ::2] = 3e38; z[6, 1::2] = -3e38
    tok = torch.from_numpy(r.integers(0, V, 7)).to(torch.int32)
    top = min(V, 5)
    o, w = forward(z, tok, temperature, top), L.token_logprob(to_np(z), tok.numpy(), t, top)
    np.testing.assert_array_equal(o["top_ids"].cpu().numpy(), w["top_ids"])
    with np.errstate(over="ignore"):
        for k in ("logp", "entropy", "lse", "top_logp"):
            same(o[k], w[k].astype(np.float32), k)


@pytest.mark.gpu
def test_every_output_alone_leading_axes_and_wide_tokens():
    z, tok, _ = scores(24, 1003, BF16, 3)
    o = forward(z, tok, 1.0, 4)
    zd = z.view(2, 3, 4, 1003).to(DEV)
    t64 = tok.view(2, 3, 4).long().to(DEV)
    t64[0, 0, 1] = 1 << 40                               # wider than an i32: names no class
    lead = (2, 3, 4)
    for k in ("logp", "entropy", "lse", "top"):
        out = Guarded(lead, F32, DEV)
        a = dict(logp=None, entropy=None, lse=None)
        tl = ti = None
        if k == "top":
            tl, ti = Guarded((*lead, 4), F32, DEV), Guarded((*lead, 4), torch.int32, DEV)
        else:
            a[k] = out.t
        B.relay_token_logprob(zd, t64 if k == "logp" else None, 1.0, a["logp"], a["entropy"], a["lse"], tl and tl.t, ti and ti.t)
        torch.cuda.synchronize()
        if k == "top":
            assert torch.equal(tl.check().view(24, 4), o["top_logp"]) and torch.equal(ti.check().view(24, 4), o["top_ids"])
        else:
            got = out.check().view(24)
            if k == "logp":
                assert float(got[1]) == 0.0
                got[1] = o[k][1]
            assert torch.equal(got, o[k])
    one = forward(z[5], tok[5].view(()), 1.0, 4)         # rank 1: the row vectors are scalars
    assert all(torch.equal(one[k], o[k][5]) for k in o)


@pytest.mark.gpu
def test_gradient_against_differences_of_the_forward_call():
    """A direction in fp32 scores; a step of 1e-2 leaves an error of its square, fp32 results one of 1e-7 / 1e-2."""
    N, V = 6, 700
    z, tok, r = scores(N, V, F32, 44)
    dlogp, dent = r.normal(size=N), r.normal(size=N)
    v = torch.from_numpy(r.normal(size=(N, V))).float()

    def scalar(x):
        o = forward(x, tok, 0.9)
        return float((to_np(o["logp"]) * dlogp).sum() + (to_np(o["entropy"]) * dent).sum())

    o = forward(z, tok, 0.9)
    dz = torch.empty(N, V, device=DEV)
    B.relay_token_logprob_grad(z.to(DEV), tok.to(DEV), 0.9, o["lse"], o["entropy"], torch.from_numpy(dlogp).float().to(DEV),
                               torch.from_numpy(dent).float().to(DEV), dz)
    an = float((to_np(dz) * to_np(v)).sum())
    fd = (scalar(z + 1e-2 * v) - scalar(z - 1e-2 * v)) / 2e-2
    assert abs(fd - an) <= 2e-3 * max(1.0, abs(an)), (fd, an)
    np.testing.assert_allclose(to_np(dz).sum(1), 0, atol=1e-5)


@pytest.mark.gpu
def test_same_bits_every_time_and_on_another_stream():
    for N, V in [(1, 131072), (40, 20011), (700, 5000)]:
        z, tok, _ = scores(N, V, BF16, 50 + N)
        o = forward(z, tok, 1.0, 10)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(3):
                again = forward(z, tok, 1.0, 10)
                assert all(torch.equal(o[k], again[k]) for k in o)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """Rows behind the 2^31st score: a few rows with one class far above the others."""
    N, V = 70001, 32768
    z = torch.zeros(N, V, dtype=BF16, device=DEV)
    hot = torch.tensor([0, 1, 65535, 65536, 69999, 70000], device=DEV)
    z[hot, (hot * 7) % V] = 20.0
    tok = ((torch.arange(N, device=DEV) * 7) % V).to(torch.int32)
    logp, ent = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    lse, tl, ti = torch.empty(N, device=DEV), torch.empty(N, 1, device=DEV), torch.empty(N, 1, dtype=torch.int32, device=DEV)
    B.relay_token_logprob(z, tok, 1.0, logp, ent, lse, tl, ti)
    want = torch.zeros(N, dtype=torch.int32, device=DEV)
    want[hot] = tok[hot]
    assert torch.equal(ti[:, 0], want)
    assert float((logp[hot] - (20 - np.log(np.exp(20.0) + V - 1))).abs().max()) < 1e-4
    dz = torch.empty_like(z)
    B.relay_token_logprob_grad(z, tok, 1.0, lse, None, torch.ones(N, device=DEV), None, dz)
    rows = torch.tensor([0, 65536, 70000, 66000], device=DEV)
    p = torch.softmax(z[rows].float(), 1)
    g = -p
    g[torch.arange(4), tok[rows].long()] += 1
    assert float((dz[rows].float() - g).abs().max()) < 4e-3


@pytest.mark.gpu
def test_no_rows():
    z, e = torch.zeros(0, 5, device=DEV), torch.zeros(0, device=DEV)
    B.relay_token_logprob(z, e.int(), 1.0, e, e.clone(), e.clone(), torch.zeros(0, 2, device=DEV), torch.zeros(0, 2, dtype=torch.int32, device=DEV))
    B.relay_token_logprob_grad(z, e.int(), 1.0, e, None, e, None, z.clone())


def test_refusals_leave_outputs_untouched(monkeypatch):
    """Everything here is refused on the host, before a launch; the tensors are host memory."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    z, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    v = lambda *s, dt=F32: torch.full(s, 5, dtype=dt)
    lp, en, ls, tl, ti, dz = v(4), v(4), v(4), v(4, 3), v(4, 3, dt=torch.int32), v(4, 8)
    f, g = B.relay_token_logprob, B.relay_token_logprob_grad
    cases = [(lambda: f(z, None, 1.0, lp, en, ls), "ERR_NULL"),
             (lambda: f(z, t, 1.0, None, en, ls), "ERR_NULL"),
             (lambda: f(z, t, 1.0, lp, en, ls, tl, None), "ERR_NULL"),
             (lambda: f(z, None, 1.0, None, None, None), "ERR_NULL"),
             (lambda: f(torch.zeros(()), None, 1.0, None, en, None), "ERR_RANK"),
             (lambda: f(z, t.view(4, 1), 1.0, lp, en, ls), "ERR_RANK"),
             (lambda: f(z, t, 1.0, lp, en, ls, v(3), ti), "ERR_RANK"),
             (lambda: f(z.int(), t, 1.0, lp, en, ls), "ERR_DTYPE"),
             (lambda: f(z, t.float(), 1.0, lp, en, ls), "ERR_DTYPE"),
             (lambda: f(z, t, 1.0, lp.bfloat16(), en, ls), "ERR_DTYPE"),
             (lambda: f(z, t, 1.0, lp, en, ls, tl, ti.long()), "ERR_DTYPE"),
             (lambda: f(torch.zeros(4, 0), t, 1.0, lp, en, ls), "ERR_SHAPE"),
             (lambda: f(z, t[:3].contiguous(), 1.0, lp, en, ls), "ERR_SHAPE"),
             (lambda: f(z, t, 1.0, lp, en, ls, v(4, 2), ti), "ERR_SHAPE"),
             (lambda: f(z, t, 1.0, lp, en, ls, v(4, 9), v(4, 9, dt=torch.int32)), "ERR_SHAPE"),      # more than there are
             (lambda: f(torch.zeros(4, 99), t, 1.0, lp, en, ls, v(4, 65), v(4, 65, dt=torch.int32)), "ERR_SHAPE"),
             (lambda: f(z, t, 0.0, lp, en, ls), "ERR_ATTR"),
             (lambda: f(z, t, -1.0, lp, en, ls), "ERR_ATTR"),
             (lambda: f(z, t, NAN, lp, en, ls), "ERR_ATTR"),
             (lambda: f(z, t, INF, lp, en, ls), "ERR_ATTR"),
             (lambda: f(z, t, 1.0, lp, lp, ls), "ERR_ATTR"),
             (lambda: f(torch.zeros(33)[1:].view(4, 8), t, 1.0, lp, en, ls), "ERR_ALIGN"),
             (lambda: g(z, None, 1.0, ls, None, lp, None, dz), "ERR_NULL"),
             (lambda: g(z, t, 1.0, ls, None, lp, en, dz), "ERR_NULL"),
             (lambda: g(z, t, 1.0, ls, None, lp, None, dz.bfloat16()), "ERR_DTYPE"),
             (lambda: g(z, t, 1.0, ls, None, v(5), None, dz), "ERR_SHAPE"),
             (lambda: g(z, t, 1.0, ls, None, lp, None, v(4, 7)), "ERR_SHAPE"),
             (lambda: g(z, t, 0.0, ls, None, lp, None, dz), "ERR_ATTR"),
             (lambda: g(z, t, 1.0, ls, None, lp, None, z), "ERR_ATTR")]
    n0 = B.relay_launch_count()
    for i, (call, status) in enumerate(cases):
        with pytest.raises(B.RelayError) as e:
            call()
        assert e.value.status_name == status, (i, e.value)
    assert B.relay_launch_count() == n0
    for x in (lp, en, ls, tl, ti, dz):
        assert bool((x == 5).all())
