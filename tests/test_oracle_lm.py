"""The float64 definitions of the language-model operators (oracle/lm.py)
against finite differences, identities and an independent dense form."""
import numpy as np
import pytest

from oracle import lm


def test_rotary_is_a_rotation_and_inverse_undoes_it():
    rng = np.random.default_rng(5)
    x = rng.standard_normal((7, 3, 10))
    pos, freqs = np.array([0, 1, -5, 1000, 10 ** 6, 3, 2 ** 33]), 10.0 ** -np.arange(4)
    for inter in (False, True):
        y = lm.rotary(x, pos, freqs, inter, False, 2.0)
        assert np.allclose((y[..., :8] ** 2).sum(-1), 4 * (x[..., :8] ** 2).sum(-1))
        assert np.array_equal(y[..., 8:], x[..., 8:])
        assert np.allclose(y[0, :, :8], 2 * x[0, :, :8])          # position 0
        back = lm.rotary(y, pos, freqs, inter, True, 0.5)
        assert np.allclose(back, x, atol=1e-9)
        # the inverse is the transpose: <y(x), e> = <x, inverse(e)>
        e = rng.standard_normal(x.shape)
        f = lm.rotary(e, pos, freqs, inter, True, 2.0)
        assert np.isclose((y * e).sum(), (x * f).sum())
    # scores of rotated queries and keys depend on the positions' difference
    q, k = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8))
    s = [(lm.rotary(q, [a + 11], freqs) * lm.rotary(k, [a], freqs)).sum() for a in (0, 5, 400)]
    assert np.allclose(s, s[0])


@pytest.mark.parametrize("causal", [False, True])
def test_attention_gradient_is_the_difference_quotient(causal):
    rng = np.random.default_rng(6)
    cu_q, cu_k = [0, 3, 3, 8], [0, 4, 6, 9]                         # one sequence has no query
    q, k, v = (rng.standard_normal((n, h, 3)) for n, h in ((8, 4), (9, 2), (9, 2)))
    e = rng.standard_normal(q.shape)
    full = lm.attention(q, k, v, cu_q, cu_k, causal, 0.7, e)

    def loss(q, k, v):
        return (lm.attention(q, k, v, cu_q, cu_k, causal, 0.7)["o"] * e).sum()
    for n, x in (("dq", q), ("dk", k), ("dv", v)):
        args = dict(q=q, k=k, v=v)
        for _ in range(25):
            at = tuple(rng.integers(0, s) for s in x.shape)
            vals = []
            for d in (1e-5, -1e-5):
                y = x.copy()
                y[at] += d
                vals.append(loss(**{**args, n[1]: y}))
            assert np.isclose((vals[0] - vals[1]) / 2e-5, full[n][at], rtol=1e-6, atol=1e-8)
    # the sequence without queries leaves its keys without gradient
    assert (full["dk"][4:6] == 0).all() and (full["dv"][4:6] == 0).all()


def test_attention_against_a_dense_form_and_empty_rows():
    rng = np.random.default_rng(7)
    q, k, v = rng.standard_normal((6, 1, 5)), rng.standard_normal((4, 1, 5)), rng.standard_normal((4, 1, 5))
    r = lm.attention(q, k, v, [0, 6], [0, 4], True, 0.3)
    S = 0.3 * q[:, 0] @ k[:, 0].T
    S[np.arange(4)[None] > np.arange(6)[:, None] - 2] = -np.inf
    with np.errstate(invalid="ignore", divide="ignore"):
        P = np.exp(S - np.where(np.isfinite(S.max(1)), S.max(1), 0)[:, None])
        o = np.where(P.sum(1)[:, None] > 0, P @ v[:, 0] / P.sum(1)[:, None], 0)
        lse = np.log(np.exp(S).sum(1))
    assert np.allclose(r["o"][:, 0], o) and np.allclose(r["lse"][0], lse)
    assert (r["o"][:2] == 0).all() and np.isneginf(r["lse"][0, :2]).all()


def test_distill_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(8)
    z = rng.standard_normal((5, 11)) * 2
    idx = np.array([[0, 3, 10], [2, 2, 5], [7, -1, 11], [1, 4, 6], [-1, -1, -1]])
    t = rng.standard_normal((5, 3))
    w = np.array([1.0, 0.5, 2.0, 0.0, 1.0])
    loss, g, _, _ = lm.distill(z, idx, t, w, 1.7, 3.0)
    assert loss[3] == 0 and loss[4] == 0 and (g[3:] == 0).all()
    assert np.allclose(g.sum(1), 0)
    for _ in range(40):
        n, j = rng.integers(0, 3), rng.integers(0, 11)
        d = []
        for h in (1e-5, -1e-5):
            y = z.copy()
            y[n, j] += h
            d.append(lm.distill(y, idx, t, w, 1.7, 3.0)[0].sum())
        assert np.isclose(3.0 * (d[0] - d[1]) / 2e-5, g[n, j], rtol=1e-6, atol=1e-9)
    # a student equal to the teacher on its entries and -Inf elsewhere: no loss
    z = np.full((1, 11), -np.inf)
    z[0, [0, 3, 10]] = t[0]
    loss, g, _, _ = lm.distill(z, idx[:1], t[:1], w[:1], 1.7, 1.0)
    assert abs(loss[0]) < 1e-12 and np.abs(g).max() < 1e-12
