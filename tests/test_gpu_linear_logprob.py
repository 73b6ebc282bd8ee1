"""GPU parity: log-probabilities from the head's operands and their gradient group against the fp64 definitions, through the C ABI.

Tolerances.  Scores are exact products of the stored operands summed in fp32 (f32 operands: to 1e-7 of their RMS), so lse and logp, sums and
differences of numbers of the size of the scores, are held to 2e-5 of that size.  The gradients are held to the sums M of their terms'
absolute values, of a token's 1 - p the one and the p (lse is an fp32 number: the difference cannot be better than its last place).  With eps = 2^-24: a partial of a score is exp(z - lse), off by the roundings of z and lse (below 64 here, so at most 64 eps
each, and as much for the sums behind z and the exponential), and the sums of fp32 products add 256 more at most: 512 eps M.  With bf16
operands the partials are rounded to bf16 before the products, by half a step, 2^-8 of each at most, so by 2^-8 M, and the results once by half
a unit in the last place."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import state_space as S
from paper_1810_00952_b200 import binding as B

from parity import Guarded, bf16_ulp, rms, to_np, workspace

DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def make(N, K, V, dt, seed, tied=False, i64=False, padded=True):
    r = np.random.default_rng(seed)
    w = r.normal(size=(K, V)) * 1.5 / np.sqrt(K)
    tokens = r.integers(0, V, N)
    x = r.normal(size=(N, K)) + 3.0 * (r.random((N, 1)) < 0.5) * w.T[tokens]
    if padded and N > 2:
        tokens[r.random(N) < 0.2] = -1
        tokens[N // 2] = V                                 # names no class either
    return dict(x=torch.from_numpy(x).to(dt), w=torch.from_numpy(w.T.copy() if tied else w).to(dt), tokens=torch.from_numpy(tokens).to(torch.int64 if i64 else torch.int32),
                dlogp=torch.from_numpy(r.normal(size=N)).float(), tied=tied)


def plain_w(t):
    return to_np(t["w"]).T if t["tied"] else to_np(t["w"])


def forward(t, temperature):
    N = t["x"].shape[0]
    logp, lse = Guarded((N,), F32, DEV), Guarded((N,), F32, DEV)
    x, w = t["x"].to(DEV), t["w"].to(DEV)
    ws = workspace(B.relay_workspace_bytes_linear_logprob(x, w, t["tied"]), DEV).fill_(0xFF)
    B.relay_linear_logprob(x, w, t["tied"], t["tokens"].to(DEV), temperature, logp.t, lse.t, ws)
    torch.cuda.synchronize()
    return logp.check(all_written=False), lse.check(all_written=False)


def gradient(t, temperature, lse, dx=True, dw=True):
    x, w = t["x"].to(DEV), t["w"].to(DEV)
    gx, gw = Guarded(tuple(x.shape), x.dtype, DEV), Guarded(tuple(w.shape), w.dtype, DEV)
    ws = workspace(B.relay_workspace_bytes_linear_logprob_grad(x, w, t["tied"]), DEV).fill_(0xFF)
    B.relay_linear_logprob_grad(x, w, t["tied"], t["tokens"].to(DEV), temperature, lse, t["dlogp"].to(DEV), gx.t if dx else None, gw.t if dw else None, ws)
    torch.cuda.synchronize()
    return gx.check() if dx else None, gw.check() if dw else None


def check(t, temperature=1.0):
    tokens = t["tokens"].tolist()
    logp, lse = forward(t, temperature)
    wl, ws = S.linear_logprob(to_np(t["x"]), plain_w(t), tokens, temperature)
    size = 1.0 + np.abs(ws).max()
    assert np.abs(to_np(lse) - ws).max() <= 2e-5 * size and np.abs(to_np(logp) - wl).max() <= 2e-5 * (size + np.abs(wl).max())
    assert all(float(v) == 0.0 for v, k in zip(logp, tokens) if not 0 <= k < plain_w(t).shape[1])
    dx, dw = gradient(t, temperature, lse)
    wx, ww = S.linear_logprob_grad(to_np(t["x"]), plain_w(t), tokens, temperature, ws, to_np(t["dlogp"]))
    sx, sw = S.linear_logprob_grad(to_np(t["x"]), plain_w(t), tokens, temperature, ws, to_np(t["dlogp"]), sizes=True)
    within(dx, wx, sx, "dx"); within(dw, ww.T if t["tied"] else ww, sw.T if t["tied"] else sw, "dw")


def within(got, want, size, what):
    g = to_np(got)
    assert g.shape == want.shape and np.all(np.isfinite(g)), what
    bound = 512 * 2.0 ** -24 * size + 1e-37
    if got.dtype == BF16:
        bound += 2.0 ** -8 * size + 0.5 * bf16_ulp(want) * (1 + 2.0 ** -7)
        assert rms(g - want) <= 4e-3 * rms(want) + 1e-37, (what, rms(g - want) / rms(want))   # of roundings that are not all at their worst
    worst = (np.abs(g - want) / bound).max() if g.size else 0.0
    assert worst <= 1.0, (what, float(worst))


SHAPES = [(1, 64, 1000), (5, 72, 333), (64, 128, 512), (33, 100, 257), (130, 64, 1029), (300, 200, 640), (257, 96, 2056), (16, 8, 40), (3, 1, 1), (70, 24, 7)]


@pytest.mark.gpu
@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_parity(shape, dt, tied):
    N, K, V = shape
    check(make(N, K, V, dt, seed=N + V, tied=tied, i64=N % 2 == 0), 1.0 if N % 2 else 0.7)


def check64(t, logp, lse, dx, dw, temperature=1.0):
    """The same comparisons with torch's 64-bit products, for sizes that take NumPy minutes."""
    x, w, dlogp, tokens = (t[k].to(DEV) for k in ("x", "w", "dlogp", "tokens"))
    x, w, dlogp, tokens = x.double(), (w.T if t["tied"] else w).double(), dlogp.double(), tokens.long()
    V = w.shape[1]
    real = (tokens >= 0) & (tokens < V)
    z = (x @ w) / temperature
    want = torch.logsumexp(z, 1)
    assert float((lse.double() - want).abs().max()) <= 2e-5 * (1 + float(want.abs().max()))
    rows, at = torch.arange(len(x), device=DEV), tokens.clamp(0, V - 1)
    wl = torch.where(real, z[rows, at] - want, 0.0)
    assert float((logp.double() - wl).abs().max()) <= 2e-5 * (1 + float(want.abs().max()) + float(wl.abs().max()))
    slope = torch.where(real, dlogp, 0.0) / temperature
    dz = -slope[:, None] * torch.exp(z - want[:, None])
    size = dz.abs()
    size[rows, at] += slope.abs()
    dz[rows, at] += slope
    flip = (lambda v: v.T) if t["tied"] else (lambda v: v)
    within(dx, to_np(dz @ w.T), to_np(size @ w.T.abs()), "dx")
    within(dw, to_np(flip(x.T @ dz)), to_np(flip(x.T.abs() @ size)), "dw")


@pytest.mark.gpu
@pytest.mark.parametrize("tied,K", [(False, 256), (True, 264), (False, 2112), (True, 2112)])
def test_many_tiles(tied, K):
    """More row blocks and columns than pairs of SMs; contractions on both sides of the length from which units are wider."""
    t = make(700, K, 9000, BF16, seed=K, tied=tied)
    logp, lse = forward(t, 1.0)
    check64(t, logp, lse, *gradient(t, 1.0, lse))


@pytest.mark.gpu
def test_leading_axes_are_rows():
    t = make(24, 40, 100, F32, seed=2)
    logp, lse = forward(t, 1.0)
    x, w, ws = t["x"].to(DEV).view(2, 3, 4, 40), t["w"].to(DEV), workspace(1 << 20, DEV)
    l2, s2 = torch.empty(2, 3, 4, device=DEV), torch.empty(2, 3, 4, device=DEV)
    tokens = t["tokens"].to(DEV).view(2, 3, 4)
    B.relay_linear_logprob(x, w, False, tokens, 1.0, l2, s2, ws)
    assert torch.equal(l2.view(-1), logp) and torch.equal(s2.view(-1), lse)
    row = torch.empty((), device=DEV)
    B.relay_linear_logprob(x[0, 0, 0], w, False, tokens[0, 0, 0].clone(), 1.0, row, torch.empty((), device=DEV), ws)
    assert abs(float(row) - float(logp[0])) <= 1e-5
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    ws = workspace(B.relay_workspace_bytes_linear_logprob_grad(x, w, False), DEV)
    B.relay_linear_logprob_grad(x, w, False, tokens, 1.0, s2, t["dlogp"].to(DEV).view(2, 3, 4), dx, dw, ws)
    want = gradient(t, 1.0, lse)
    assert torch.equal(dx.view(24, 40), want[0]) and torch.equal(dw, want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_one_gradient_alone_is_the_same(dt):
    t = make(90, 72, 500, dt, seed=3, tied=dt == BF16)
    _, lse = forward(t, 1.3)
    dx, dw = gradient(t, 1.3, lse)
    assert torch.equal(gradient(t, 1.3, lse, dw=False)[0], dx) and torch.equal(gradient(t, 1.3, lse, dx=False)[1], dw)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_rows_without_a_token_take_no_part_whatever_they_hold(dt):
    t = make(80, 64, 320, dt, seed=4, padded=False)
    t["tokens"][::3] = -1
    clean = forward(t, 1.0)
    want = gradient(t, 1.0, clean[1])
    bad = torch.zeros(80, dtype=torch.bool)
    bad[::6] = True
    t["x"][bad] = float("nan")
    t["dlogp"][::3] = float("inf")
    logp, lse = forward(t, 1.0)
    assert torch.equal(logp, clean[0]) and torch.equal(lse.cpu()[~bad], clean[1].cpu()[~bad]) and bool(torch.isnan(lse.cpu()[bad]).all())
    got = gradient(t, 1.0, lse)
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and not bool(got[0][::3].any())


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_infinite_scores(dt):
    x = torch.tensor([[1.0, 0.0], [-1.0, 0.0], [0.5, 1.0]], dtype=dt)
    w = torch.randn(2, 300, generator=torch.Generator().manual_seed(1)).to(dt)
    t = dict(x=x, w=w.clone(), tokens=torch.tensor([5, 6, 7], dtype=torch.int32), dlogp=torch.ones(3), tied=False)
    t["w"][0, 100:] = -float("inf")                        # classes that cannot occur for the first and third row; +inf for the second
    t["w"][1, 100:] = 0.0
    t["x"][:, 1] = 1.0
    logp, lse = forward(t, 1.0)
    if dt == F32:                                          # the compensated sums of the fp32 contraction know no infinities
        assert bool(torch.isnan(lse).all()) and bool(torch.isnan(logp).all())
        return
    wl, ws = S.linear_logprob(to_np(t["x"]), to_np(t["w"]), [5, 6, 7], 1.0)
    np.testing.assert_allclose(to_np(lse)[[0, 2]], ws[[0, 2]], rtol=2e-5); np.testing.assert_allclose(to_np(logp)[[0, 2]], wl[[0, 2]], rtol=2e-5)
    assert np.isnan(to_np(lse)[1]) and np.isnan(to_np(logp)[1])
    t["w"][0, :] = -float("inf")                           # nothing can occur
    logp, lse = forward(t, 1.0)
    assert all(np.isneginf(to_np(v)[[0, 2]]).all() for v in (logp, lse))


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [BF16, F32])
def test_a_nearly_certain_token_keeps_its_slope(dt):
    """p = 1 - 3e-6: dlogp (1 - p) comes from the logarithm, not from 1 - p."""
    K, V = 64, 200
    w = torch.zeros(K, V)
    w[0, 9] = 1.0
    x = torch.zeros(70, K)
    x[:, 0] = 18.0
    t = dict(x=x.to(dt), w=w.to(dt), tokens=torch.full((70,), 9, dtype=torch.int32), dlogp=torch.ones(70), tied=False)
    logp, lse = forward(t, 1.0)
    wl, ws = S.linear_logprob(to_np(t["x"]), to_np(t["w"]), [9] * 70, 1.0)
    dx, dw = gradient(t, 1.0, torch.from_numpy(ws).float().to(DEV))
    wx, ww = S.linear_logprob_grad(to_np(t["x"]), to_np(t["w"]), [9] * 70, 1.0, to_np(torch.from_numpy(ws).float()), np.ones(70))
    # lse is stored with 2^-24 of 18, 1e-6: that much of one, a third of 1 - p, lies in what is given, not in the call
    rel = 2.0 ** -8 if dt == BF16 else 1e-4
    assert abs(float(dw[0, 9]) - ww[0, 9]) <= (rel + 1e-3) * abs(ww[0, 9])


@pytest.mark.gpu
def test_pieces_of_the_vocabulary_join():
    """N x V above what a piece holds (2^27): several pieces, the last one of odd size and copied; dx is summed over them."""
    for dt, N, K, V, tied in ((BF16, 4096, 64, 70001, False), (BF16, 4096, 64, 70001, True), (F32, 2048, 16, 70001, False)):
        g = torch.Generator(device=DEV).manual_seed(5)
        x = torch.randn(N, K, generator=g, device=DEV).to(dt)
        w = (0.3 * torch.randn((V, K) if tied else (K, V), generator=g, device=DEV)).to(dt)
        tokens = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
        tokens[:4] = torch.tensor([0, V - 1, V - 2, 32768], dtype=torch.int32)
        dlogp = torch.randn(N, generator=g, device=DEV)
        logp, lse = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
        B.relay_linear_logprob(x, w, tied, tokens, 1.0, logp, lse, workspace(B.relay_workspace_bytes_linear_logprob(x, w, tied), DEV))
        dx, dw = Guarded((N, K), dt, DEV), Guarded(tuple(w.shape), dt, DEV)
        need = B.relay_workspace_bytes_linear_logprob_grad(x, w, tied)
        assert need < N * V * (2 if dt == BF16 else 4)     # less than the scores
        B.relay_linear_logprob_grad(x, w, tied, tokens, 1.0, lse, dlogp, dx.t, dw.t, workspace(need, DEV).fill_(0xFF))
        check64(dict(x=x, w=w, tokens=tokens, dlogp=dlogp, tied=tied), logp, lse, dx.check(), dw.check())
    B.relay_poll_status()


@pytest.mark.gpu
def test_no_rows():
    t = make(0, 16, 30, F32, seed=7)
    forward(t, 1.0)
    _, dw = gradient(t, 1.0, torch.empty(0, device=DEV))
    assert not bool(dw.any())


def test_refusals_leave_outputs_untouched(monkeypatch):
    """Everything here is refused on the host, before a launch; the tensors are host memory."""
    monkeypatch.setattr(B, "_stream", lambda: ctypes.c_void_p(None))
    z = lambda *s, dt=F32: torch.zeros(*s, dtype=dt)
    x, w, tok, one = z(6, 16), z(16, 40), z(6, dt=torch.int32), z(6)
    logp, lse, dx, dw = (torch.full(s, 5.0) for s in ((6,), (6,), (6, 16), (16, 40)))
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    f, g = B.relay_linear_logprob, B.relay_linear_logprob_grad
    cases = [(lambda: f(None, w, 0, tok, 1.0, logp, lse, ws), "ERR_NULL"), (lambda: f(x, w, 0, None, 1.0, logp, lse, ws), "ERR_NULL"),
             (lambda: f(x, w, 0, tok, 1.0, None, lse, ws), "ERR_NULL"), (lambda: f(x, w, 0, tok, 1.0, logp, None, ws), "ERR_NULL"),
             (lambda: f(x, w[0], 0, tok, 1.0, logp, lse, ws), "ERR_RANK"), (lambda: f(z(()), w, 0, tok, 1.0, logp, lse, ws), "ERR_RANK"),
             (lambda: f(x, w, 0, z(6, 1, dt=torch.int32), 1.0, logp, lse, ws), "ERR_RANK"),
             (lambda: f(x, w.bfloat16(), 0, tok, 1.0, logp, lse, ws), "ERR_DTYPE"), (lambda: f(x, w, 0, one, 1.0, logp, lse, ws), "ERR_DTYPE"),
             (lambda: f(x, w, 0, tok, 1.0, logp.bfloat16(), lse, ws), "ERR_DTYPE"),
             (lambda: f(x, w, 1, tok, 1.0, logp, lse, ws), "ERR_SHAPE"), (lambda: f(x, z(15, 40), 0, tok, 1.0, logp, lse, ws), "ERR_SHAPE"),
             (lambda: f(x, z(16, 0), 0, tok, 1.0, logp, lse, ws), "ERR_SHAPE"), (lambda: f(z(6, 0), z(0, 40), 0, tok, 1.0, logp, lse, ws), "ERR_SHAPE"),
             (lambda: f(x, w, 0, z(5, dt=torch.int32), 1.0, logp, lse, ws), "ERR_SHAPE"),
             (lambda: f(x, w, 0, tok, 0.0, logp, lse, ws), "ERR_ATTR"), (lambda: f(x, w, 0, tok, -1.0, logp, lse, ws), "ERR_ATTR"),
             (lambda: f(x, w, 0, tok, float("nan"), logp, lse, ws), "ERR_ATTR"), (lambda: f(x, w, 0, tok, float("inf"), logp, lse, ws), "ERR_ATTR"),
             (lambda: f(x, w, 0, tok, 1.0, logp, logp, ws), "ERR_ATTR"),
             (lambda: f(z(97)[1:].view(6, 16), w, 0, tok, 1.0, logp, lse, ws), "ERR_ALIGN"),
             (lambda: f(x, w, 0, tok, 1.0, logp, lse, None), "ERR_WORKSPACE"), (lambda: f(x, w, 0, tok, 1.0, logp, lse, ws[:16]), "ERR_WORKSPACE"),
             (lambda: f(x, w, 0, tok, 1.0, logp, lse, ws[8:]), "ERR_WORKSPACE"),
             (lambda: g(x, w, 0, tok, 1.0, one, one, None, None, ws), "ERR_NULL"), (lambda: g(x, w, 0, tok, 1.0, None, one, dx, dw, ws), "ERR_NULL"),
             (lambda: g(x, w, 0, tok, 1.0, one, None, dx, dw, ws), "ERR_NULL"),
             (lambda: g(x, w, 0, tok, 1.0, one, one, dx.bfloat16(), dw, ws), "ERR_DTYPE"), (lambda: g(x, w, 0, tok, 1.0, one.double().to(BF16), one, dx, dw, ws), "ERR_DTYPE"),
             (lambda: g(x, w, 0, tok, 1.0, one, one, dx, z(40, 16), ws), "ERR_SHAPE"), (lambda: g(x, w, 0, tok, 1.0, one, z(7), dx, dw, ws), "ERR_SHAPE"),
             (lambda: g(x, w, 0, tok, 1.0, one, one, x, dw, ws), "ERR_ATTR"), (lambda: g(x, w, 0, tok, 1.0, one, one, dx, w, ws), "ERR_ATTR"),
             (lambda: g(x, w, 0, tok, 1.0, one, one, dx, dw, ws[:64]), "ERR_WORKSPACE")]
    n0 = B.relay_launch_count()
    for i, (call, status) in enumerate(cases):
        with pytest.raises(B.RelayError) as e:
            call()
        assert e.value.status_name == status, (i, e.value)
    assert B.relay_launch_count() == n0
    assert all(bool((t == 5).all()) for t in (logp, lse, dx, dw))
    assert B.relay_workspace_bytes_linear_logprob(x, w, 1) == 0 and B.relay_workspace_bytes_linear_logprob_grad(x, z(15, 40), 0) == 0


@pytest.mark.gpu
def test_more_rows_than_one_slab_of_statistics():
    """2^28 bytes of statistics are 33,280 rows of 64,100 classes (1,004 statistics of 8 bytes a row, whole tiles of 256 rows): the rows behind them come in a second slab."""
    N, K, V = 34000, 64, 64100
    g = torch.Generator(device=DEV).manual_seed(8)
    x, w = torch.randn(N, K, generator=g, device=DEV).to(BF16), (0.2 * torch.randn(V, K, generator=g, device=DEV)).to(BF16)
    tokens = torch.randint(0, V, (N,), generator=g, device=DEV)
    logp, lse = Guarded((N,), F32, DEV), Guarded((N,), F32, DEV)
    need = B.relay_workspace_bytes_linear_logprob(x, w, True)
    assert need < 3 << 27
    B.relay_linear_logprob(x, w, True, tokens, 1.0, logp.t, lse.t, workspace(need, DEV).fill_(0xFF))
    logp, lse = logp.check(), lse.check()
    for rows in (slice(0, 300), slice(33000, N)):
        z = x[rows].double() @ w.double().T
        want = torch.logsumexp(z, 1)
        assert float((lse[rows].double() - want).abs().max()) <= 2e-5 * (1 + float(want.abs().max()))
        at = z.gather(1, tokens[rows, None])[:, 0] - want
        assert float((logp[rows].double() - at).abs().max()) <= 2e-5 * (1 + 2 * float(want.abs().max()) + float(at.abs().max()))
    B.relay_poll_status()


@pytest.mark.gpu
def test_more_rows_than_one_slab_of_scores():
    """f32: 2^27 scores are 524,288 rows of 256 classes, the smallest piece; the rows behind them come in a second slab."""
    N, K, V = 525000, 8, 300
    g = torch.Generator(device=DEV).manual_seed(9)
    x, w = torch.randn(N, K, generator=g, device=DEV), torch.randn(K, V, generator=g, device=DEV)
    tokens = torch.randint(0, V, (N,), generator=g, device=DEV)
    logp, lse = Guarded((N,), F32, DEV), Guarded((N,), F32, DEV)
    need = B.relay_workspace_bytes_linear_logprob(x, w, False)
    assert need < 5 << 27                                   # 2^27 scores of 4 bytes and a little
    B.relay_linear_logprob(x, w, False, tokens, 1.0, logp.t, lse.t, workspace(need, DEV).fill_(0xFF))
    logp, lse = logp.check(), lse.check()
    for rows in (slice(0, 300), slice(524000, N)):
        z = x[rows].double() @ w.double()
        want = torch.logsumexp(z, 1)
        assert float((lse[rows].double() - want).abs().max()) <= 2e-5 * (1 + float(want.abs().max()))
        at = z.gather(1, tokens[rows, None])[:, 0] - want
        assert float((logp[rows].double() - at).abs().max()) <= 2e-5 * (1 + 2 * float(want.abs().max()) + float(at.abs().max()))
    B.relay_poll_status()
