"""Pins of the oracle's definitions for state space language models: closed forms, independent routes, finite differences."""
import numpy as np
import pytest

from oracle import language as L
from oracle import state_space as S

from test_oracle_language import central


def conv_inputs(T, B, D, K, seed):
    r = np.random.default_rng(seed)
    return r.normal(size=(T, B, D)), r.normal(size=(K, D)), r.normal(size=D), r.normal(size=(K - 1, B, D)), r


def test_conv_equals_numpy_convolution_and_its_state_continues_it():
    x, w, b, before, _ = conv_inputs(9, 2, 3, 4, 1)
    y, after = S.causal_conv(x, w, b, before, None, False)
    for i in range(2):
        for d in range(3):
            line = np.concatenate([before[:, i, d], x[:, i, d]])
            np.testing.assert_allclose(y[:, i, d], np.convolve(line, w[::-1, d], "valid") + b[d], rtol=1e-12, atol=1e-12)
    first, mid = S.causal_conv(x[:5], w, b, before, None, True)
    second, last = S.causal_conv(x[5:], w, b, mid, None, True)
    whole, end = S.causal_conv(x, w, b, before, None, True)
    np.testing.assert_array_equal(np.concatenate([first, second]), whole)
    np.testing.assert_array_equal(last, end)
    np.testing.assert_array_equal(S.causal_conv(x[:0], w, b, before, None, True)[1], before)
    np.testing.assert_array_equal(S.causal_conv(x[:1], w, b, before, None, True)[1], np.concatenate([before[1:], x[:1]]))


@pytest.mark.parametrize("silu,lengths", [(False, None), (True, None), (True, [5, 0, 2])])
def test_conv_gradient_matches_differences(silu, lengths):
    x, w, b, before, r = conv_inputs(5, 3, 2, 4, 2)
    dy, dafter = r.normal(size=x.shape), r.normal(size=before.shape)
    dx, dw, db, dbefore = S.causal_conv_grad(x, w, b, before, lengths, silu, dy, dafter)

    def f():
        y, after = S.causal_conv(x, w, b, before, lengths, silu)
        return np.sum(y * dy) + np.sum(after * dafter)

    for got, arg in ((dx, x), (dw, w), (db, b), (dbefore, before)):
        np.testing.assert_allclose(got, central(f, arg), rtol=1e-6, atol=1e-8)


def scan_inputs(T, B, D, N, seed):
    r = np.random.default_rng(seed)
    t = dict(u=r.normal(size=(T, B, D)), delta=r.normal(size=(T, B, D)), a=-r.uniform(0.2, 3.0, (D, N)), b=r.normal(size=(T, B, N)),
             c=r.normal(size=(T, B, N)), d=r.normal(size=D), z=r.normal(size=(T, B, D)), delta_bias=r.normal(size=D), h0=r.normal(size=(B, D, N)))
    return t, r


def test_scan_with_one_state_is_the_gated_recurrence():
    t, _ = scan_inputs(7, 2, 3, 1, 3)
    y, h = S.selective_scan(t["u"], t["delta"], t["a"], t["b"], np.ones((7, 2, 1)), None, None, None, t["h0"], None, True)
    step = np.log1p(np.exp(t["delta"]))
    h_all, last = L.gated_recurrence(np.exp(step * t["a"][:, 0]), step * t["u"] * t["b"], t["h0"][..., 0], None, L.GATE_GIVEN)
    np.testing.assert_allclose(y, h_all, rtol=1e-12)
    np.testing.assert_allclose(h[..., 0], last, rtol=1e-12)


def test_scan_continues_from_its_state_and_lengths_cut():
    t, _ = scan_inputs(8, 3, 2, 4, 4)
    seq = [k for k in ("u", "delta", "b", "c", "z")]

    def run(s, e, h0, lengths=None):
        q = {k: (v[s:e] if k in seq else v) for k, v in t.items()}
        return S.selective_scan(q["u"], q["delta"], q["a"], q["b"], q["c"], q["d"], q["z"], q["delta_bias"], h0, lengths, True, 2)

    y, h, states = run(0, 8, t["h0"])
    y1, h1, _ = run(0, 4, t["h0"])
    y2, h2, _ = run(4, 8, h1)
    np.testing.assert_array_equal(np.concatenate([y1, y2]), y)
    np.testing.assert_array_equal(h2, h)
    np.testing.assert_array_equal(states[2], h1)
    yl, hl, sl = run(0, 8, t["h0"], [4, 0, 99])
    np.testing.assert_array_equal(yl[:4, 0], y1[:, 0]); np.testing.assert_array_equal(hl[0], h1[0]); np.testing.assert_array_equal(sl[3, 0], h1[0])
    np.testing.assert_array_equal(hl[1], t["h0"][1]); np.testing.assert_array_equal(hl[2], h[2])
    assert not yl[4:, 0].any() and not yl[:, 1].any()


@pytest.mark.parametrize("gated,softplus,bias,lengths", [(True, True, True, None), (False, False, False, None), (True, False, True, [4, 0, 2])])
def test_scan_gradient_matches_differences(gated, softplus, bias, lengths):
    t, r = scan_inputs(4, 3, 2, 3, 5)
    if not gated:
        t["z"] = t["d"] = None
    if not bias:
        t["delta_bias"] = None
    dy, dh = r.normal(size=(4, 3, 2)), r.normal(size=(3, 2, 3))
    args = lambda: [t[k] for k in ("u", "delta", "a", "b", "c", "d", "z", "delta_bias", "h0")]
    o = S.selective_scan_grad(*args(), lengths, softplus, dy, dh)

    def f():
        y, h = S.selective_scan(*args(), lengths, softplus)
        return np.sum(y * dy) + np.sum(h * dh)

    # Steps below zero let the states grow, and f with them.  f is a sum of terms of size M, rounded to about 2^-52 M times the few tens of
    # additions (square root: 8) on the way, and the quotient divides two such errors by 2 h = 2e-6: what differences leave is 8 2^-52 M / 1e-6.
    y, h = S.selective_scan(*args(), lengths, softplus)
    M = np.sum(np.abs(y * dy)) + np.sum(np.abs(h * dh))
    for k, v in t.items():
        if v is not None:
            np.testing.assert_allclose(o["d" + k], central(f, v), rtol=1e-5, atol=1e-7 + 8 * 2.0 ** -52 * M / 1e-6, err_msg=k)


def test_head_equals_the_token_log_probabilities_of_its_scores():
    r = np.random.default_rng(6)
    x, w, tokens, dlogp = r.normal(size=(5, 7)), r.normal(size=(7, 11)), np.array([3, -1, 10, 11, 0]), r.normal(size=5)
    logp, lse = S.linear_logprob(x, w, tokens, 0.7)
    want = L.token_logprob(x @ w, tokens, 0.7)
    np.testing.assert_allclose(logp, want["logp"], rtol=1e-12); np.testing.assert_allclose(lse, want["lse"], rtol=1e-12)
    dx, dw = S.linear_logprob_grad(x, w, tokens, 0.7, lse, dlogp)
    for got, arg in ((dx, x), (dw, w)):
        np.testing.assert_allclose(got, central(lambda: np.sum(S.linear_logprob(x, w, tokens, 0.7)[0] * dlogp), arg), rtol=1e-6, atol=1e-8)


def test_head_of_rows_that_have_no_softmax():
    x, w = np.array([[1.0], [-1.0], [np.nan]]), np.array([[-np.inf, -np.inf]])
    logp, lse = S.linear_logprob(x, w, np.array([0, 0, -1]), 1.0)
    assert np.isneginf(lse[0]) and np.isneginf(logp[0]) and np.isnan(lse[1]) and np.isnan(lse[2]) and logp[2] == 0.0
