"""oracle/tokens.py: the definitions against difference quotients and against
each other."""
import numpy as np

from oracle import tokens


def test_embedding_gradient_is_the_adjoint():
    rng = np.random.default_rng(1)
    tok = np.array([3, 0, 3, -1, 6, 7, 3, 0])
    e, table = rng.standard_normal((8, 5)), rng.standard_normal((7, 5))
    g, _ = tokens.embed_grad(tok, e, 7, 2.5)
    y = np.array([table[t] * 2.5 if 0 <= t < 7 else np.zeros(5) for t in tok])
    assert np.isclose((y * e).sum(), (g * table).sum(), rtol=1e-13)
    assert (g[[1, 2, 4, 5]] == 0).all()


def test_norm_and_its_gradients():
    rng = np.random.default_rng(2)
    u, w, e = rng.standard_normal((3, 6)), rng.standard_normal(6), rng.standard_normal((3, 6))
    f = lambda u, w: (tokens.norm(u, w, 0.1, 1.0, False)["y"] * e).sum()
    r = tokens.norm(u, w, 0.1, 1.0, False)
    assert np.allclose(r["y"], u / np.sqrt((u ** 2).mean(1, keepdims=True) + 0.1) * w, rtol=1e-14)
    d, _, dw, _ = tokens.norm_grad(u, w, r["rstd"], e, None)
    step = 1e-6
    for i in range(3):
        for j in range(6):
            up, down = u.copy(), u.copy()
            up[i, j] += step
            down[i, j] -= step
            assert abs((f(up, w) - f(down, w)) / (2 * step) - d[i, j]) < 1e-8
    for j in range(6):
        up, down = w.copy(), w.copy()
        up[j] += step
        down[j] -= step
        assert abs((f(u, up) - f(u, down)) / (2 * step) - dw[j]) < 1e-8
    rows = tokens.norm(u, w, 0.1, 100.0, True)
    assert np.allclose(abs(rows["y"]).max(1), 100.0)


def test_log_probabilities_and_their_gradient():
    rng = np.random.default_rng(3)
    z, idx = rng.standard_normal((4, 9)) * 2, np.array([[1, 1], [-1, 3], [8, 0], [9, -5]])
    dl, dh, tau = rng.standard_normal((4, 2)), rng.standard_normal(4), 1.7
    r = tokens.logprobs(z, idx, tau, 3)
    p = np.exp(z / tau) / np.exp(z / tau).sum(1, keepdims=True)
    assert np.allclose(r["entropy"], -(p * np.log(p)).sum(1), rtol=1e-13)
    assert np.isclose(r["logp"][0, 0], np.log(p[0, 1])) and (r["logp"][3] == 0).all()
    assert (r["top_idx"][:, 0] == z.argmax(1)).all()

    def f(z):
        r = tokens.logprobs(z, idx, tau, 0)
        return (r["logp"] * dl).sum() + (r["entropy"] * dh).sum()
    g, _ = tokens.logprobs_grad(z, idx, tau, r["stats"], r["entropy"], dl, dh, 1.0)
    step = 1e-6
    for i in range(4):
        for j in range(9):
            up, down = z.copy(), z.copy()
            up[i, j] += step
            down[i, j] -= step
            assert abs((f(up) - f(down)) / (2 * step) - g[i, j]) < 1e-8


def test_order_of_the_top():
    z = np.array([0.0, 2.0, np.nan, -0.0, 2.0, -np.inf, np.inf, np.nan])
    assert list(tokens.top_order(z)) == [2, 7, 6, 1, 4, 0, 3, 5]
