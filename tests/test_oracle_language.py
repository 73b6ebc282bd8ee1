"""Pins of the oracle's definitions for recurrent language models: closed forms, independent routes, finite differences."""
import numpy as np
import pytest

from oracle import language as L

GATES = [L.GATE_GIVEN, L.GATE_SIGMOID, L.GATE_MIX]


def central(scalar, x, h=1e-6):
    out = np.zeros_like(x)
    for k in np.ndindex(*x.shape):
        keep = x[k]
        x[k] = keep + h; up = scalar()
        x[k] = keep - h; dn = scalar()
        x[k] = keep
        out[k] = (up - dn) / (2 * h)
    return out


# ---- recurrence ----
def recurrence_inputs(T, B, D, seed):
    r = np.random.default_rng(seed)
    return r.uniform(0.2, 0.95, (T, B, D)), r.normal(size=(T, B, D)), r.normal(size=(B, D)), r


@pytest.mark.parametrize("gate", GATES)
def test_recurrence_equals_the_sum_over_all_earlier_steps(gate):
    f, u, h0, _ = recurrence_inputs(6, 2, 3, 1)
    a = f if gate == L.GATE_GIVEN else 1 / (1 + np.exp(-f))
    b = (1 - a) * u if gate == L.GATE_MIX else u
    h_all, h_final = L.gated_recurrence(f, u, h0, None, gate)
    for t in range(6):
        want = np.prod(a[:t + 1], axis=0) * h0 + sum(np.prod(a[s + 1:t + 1], axis=0) * b[s] for s in range(t + 1))
        np.testing.assert_allclose(h_all[t], want, rtol=1e-12)
    np.testing.assert_array_equal(h_all[-1], h_final)


def test_recurrence_closed_forms():
    T, B, D = 5, 2, 3
    one, x = np.ones((T, B, D)), np.random.default_rng(2).normal(size=(T, B, D))
    np.testing.assert_allclose(L.gated_recurrence(one, x, np.zeros((B, D)), None, L.GATE_GIVEN)[0], np.cumsum(x, axis=0), rtol=1e-12)
    np.testing.assert_array_equal(L.gated_recurrence(0 * one, x, one[0], None, L.GATE_GIVEN)[0], x)
    h = L.gated_recurrence(x, 3 * one, 3 * one[0], None, L.GATE_MIX)[0]            # a running mean of equal values
    np.testing.assert_allclose(h, 3.0, rtol=1e-14)
    h, last = L.gated_recurrence(60 * one, x, one[0], None, L.GATE_MIX)            # a gate that is wide open keeps its state
    np.testing.assert_allclose(last, 1.0, rtol=1e-12)


def test_recurrence_lengths_cut_each_sequence():
    f, u, h0, _ = recurrence_inputs(5, 4, 3, 3)
    f[3:, 1] = np.nan
    h_all, h_final = L.gated_recurrence(f, u, h0, [0, 3, 9, -2], L.GATE_SIGMOID)
    assert not h_all[:, 0].any() and not h_all[3:, 1].any() and not h_all[:, 3].any()
    np.testing.assert_array_equal(h_final[[0, 3]], h0[[0, 3]])
    alone = L.gated_recurrence(f[:3, 1:2], u[:3, 1:2], h0[1:2], None, L.GATE_SIGMOID)
    np.testing.assert_array_equal(alone[0], h_all[:3, 1:2]); np.testing.assert_array_equal(alone[1], h_final[1:2])
    np.testing.assert_array_equal(h_all[-1, 2], h_final[2])


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("lengths", [None, [4, 2, 0]])
def test_recurrence_gradient_matches_finite_differences(gate, lengths):
    T, B, D = 4, 3, 2
    f, u, h0, r = recurrence_inputs(T, B, D, 4)
    dh_all, dh_final = r.normal(size=(T, B, D)), r.normal(size=(B, D))
    if lengths is not None:
        for b, n in enumerate(lengths):
            dh_all[n:, b] = 0                                                     # nothing depends on the zeros behind the end

    def scalar():
        h, last = L.gated_recurrence(f, u, h0, lengths, gate)
        return float((h * dh_all).sum() + (last * dh_final).sum())

    h_all, _ = L.gated_recurrence(f, u, h0, lengths, gate)
    got = L.gated_recurrence_grad(f, u, h0, lengths, gate, h_all, dh_all, dh_final)
    for g, x in zip(got, (f, u, h0)):
        np.testing.assert_allclose(g, central(scalar, x), rtol=1e-6, atol=1e-8)


# ---- log-probabilities ----
def test_logprob_against_direct_sums_and_closed_forms():
    r = np.random.default_rng(5)
    z, tok = r.normal(size=(4, 7)), np.array([0, 6, -1, 7])
    o = L.token_logprob(z, tok, 0.5, top=3)
    p = np.exp(2 * z) / np.exp(2 * z).sum(1, keepdims=True)
    np.testing.assert_allclose(o["logp"], [np.log(p[0, 0]), np.log(p[1, 6]), 0, 0], rtol=1e-12)
    np.testing.assert_allclose(o["entropy"], -(p * np.log(p)).sum(1), rtol=1e-12)
    np.testing.assert_array_equal(o["top_ids"], np.argsort(-z, axis=1, kind="stable")[:, :3])
    o = L.token_logprob(np.full((1, 10), 4.0), np.array([3]), 1.0, top=4)
    np.testing.assert_allclose([o["logp"][0], o["entropy"][0], o["lse"][0]], [-np.log(10), np.log(10), 4 + np.log(10)], rtol=1e-13)
    np.testing.assert_array_equal(o["top_ids"][0], [0, 1, 2, 3])                   # ties: the lower id


def test_logprob_of_masked_and_non_finite_rows():
    inf, nan = np.inf, np.nan
    z = np.array([[-inf, -inf, -inf], [-inf, 1.0, -inf], [0.0, nan, 2.0], [0.0, inf, 2.0]])
    o = L.token_logprob(z, np.array([1, 1, 0, 0]), 1.0, top=2)
    assert o["lse"][0] == -inf and o["logp"][0] == -inf and o["entropy"][0] == 0 and list(o["top_ids"][0]) == [0, 1]
    assert o["logp"][1] == 0 and o["entropy"][1] == 0 and list(o["top_ids"][1]) == [1, 0] and o["top_logp"][1, 1] == -inf
    assert np.isnan(o["logp"][2:]).all() and list(o["top_ids"][2]) == [1, 2] and list(o["top_ids"][3]) == [1, 2]


@pytest.mark.parametrize("with_entropy", [False, True])
def test_logprob_gradient_matches_finite_differences(with_entropy):
    r = np.random.default_rng(6)
    z, tok = r.normal(size=(3, 5)), np.array([2, 0, -1])
    dlogp, dent = r.normal(size=3), (r.normal(size=3) if with_entropy else None)

    def scalar():
        o = L.token_logprob(z, tok, 0.7)
        return float((o["logp"] * dlogp).sum() + ((o["entropy"] * dent).sum() if with_entropy else 0))

    o = L.token_logprob(z, tok, 0.7)
    g = L.token_logprob_grad(z, tok, 0.7, o["lse"], o["entropy"], dlogp, dent)
    np.testing.assert_allclose(g, central(scalar, z), rtol=1e-6, atol=1e-9)
    np.testing.assert_allclose(g.sum(1), 0, atol=1e-12)                            # softmax does not see a shift


# ---- orthogonalisation ----
def test_orthogonalize_acts_on_the_singular_values_alone():
    r = np.random.default_rng(7)
    coef = (3.4445, -4.7750, 2.0315)
    for shape in [(6, 4), (4, 6), (5, 5), (1, 7), (7, 1)]:
        x = r.normal(size=shape)
        u, s, vt = np.linalg.svd(x, full_matrices=False)
        t = s / np.linalg.norm(x)
        for _ in range(5):
            t = coef[0] * t + coef[1] * t ** 3 + coef[2] * t ** 5
        np.testing.assert_allclose(L.orthogonalize(x, 5, coef, 0.0, 2.0), 2 * u @ np.diag(t) @ vt, rtol=1e-9, atol=1e-12)


def test_orthogonalize_converges_to_the_polar_factor_with_the_classical_coefficients():
    r = np.random.default_rng(8)
    x = r.normal(size=(2, 5, 3))
    y = L.orthogonalize(x, 40, (1.5, -0.5, 0.0), 0.0, 1.0)
    for k in range(2):
        u, _, vt = np.linalg.svd(x[k], full_matrices=False)
        np.testing.assert_allclose(y[k], u @ vt, atol=1e-10)
    assert not L.orthogonalize(np.zeros((3, 4)), 5, (3.4445, -4.775, 2.0315), 1e-7, 1.0).any()
