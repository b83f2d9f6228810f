"""Plain float64 definitions of the operators on tokens and rows, from the values
of the codes: embeddings and their gradient, the norm of a residual sum and its
gradients, log probabilities of given tokens and theirs.  Next to each result
its error bound: what FP32 arithmetic may lose before the last rounding (a sum
of n terms in any order loses (n - 1) EPS32 of the terms' magnitudes; one over a
row's W elements, which at least 64 threads share in steps of eight and join in
a tree, W / 64 + 64 terms in a chain at most).
"""
import numpy as np

EPS32 = 2.0 ** -24          # half a step of FP32, relative


def _chain(n):
    return n / 64.0 + 64.0


def embed_grad(tokens, e, V, scale):
    """e: T x W float64; returns g (V x W) and its bound."""
    g, mag, n = np.zeros((V, e.shape[1])), np.zeros((V, e.shape[1])), np.zeros(V)
    for t, v in enumerate(tokens):
        if 0 <= v < V:
            g[v] += e[t]
            mag[v] += abs(e[t])
            n[v] += 1
    return g * scale, abs(scale) * mag * (n[:, None] + 1) * EPS32


def norm(u, w, eps, y_scale, rows):
    """u: T x W float64 (the sum as stored).  Returns a dict of rstd, y and, with
    rows, scales; bounds under *_err."""
    W = u.shape[1]
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        rstd = 1.0 / np.sqrt((u * u).sum(1) / W + eps)
        rel = (_chain(W) / 2 + 6) * EPS32
        n = u * rstd[:, None] * w
        c = np.full(len(u), float(y_scale))
        if rows:
            top = abs(n).max(1)
            some = (top > 0) & np.isfinite(top)
            c = np.where(some, np.minimum(y_scale / np.where(some, top, 1), 2.0 ** 126), 1.0)
        # the norm's error cancels in a row's own scale but for the largest's
        return dict(rstd=rstd, rstd_err=rstd * rel, scales=c, scales_err=abs(c) * (rel + 4 * EPS32),
                    y=n * c[:, None], y_err=abs(n * c[:, None]) * (2 * rel + 8 * EPS32))


def norm_grad(h, w, rstd, dy, dr):
    """All float64 (dr may be None); returns d, dw and their bounds."""
    T, W = h.shape
    n, g = h * rstd[:, None], dy * w
    m = (g * n).mean(1, keepdims=True)
    m_err = (_chain(W) + 4) * EPS32 * abs(g * n).mean(1, keepdims=True)
    own = rstd[:, None] * (g - n * m)
    d = own if dr is None else dr + own
    err = rstd[:, None] * (4 * EPS32 * (abs(g) + abs(n * m)) + abs(n) * m_err) + 3 * EPS32 * abs(own)
    if dr is not None:
        err = err + EPS32 * abs(d)
    return d, err, (dy * n).sum(0), (T + 3) * EPS32 * abs(dy * n).sum(0)


def _softmax_error(d, p, V):
    """Bound of ln S: an exponent is off by 4 EPS32 of itself and as much
    again of 1, the sum by its chain."""
    return (p * 4 * EPS32 * (1 + abs(d))).sum() + (_chain(V) + 32) * EPS32


def top_order(z):
    """Indices of a row, largest first, among equals (-0 and 0) the lowest
    first, NaN above everything."""
    key = np.where(np.isnan(z), np.inf, z)
    return np.lexsort((np.arange(len(z)), -key, ~np.isnan(z)))


def logprobs(z, idx, tau, k):
    """z: N x V float64, idx: N x m.  A dict of logp, entropy, stats, top_idx,
    top_logp, and bounds under *_err."""
    N, V = z.shape
    m = idx.shape[1]
    r = dict(logp=np.zeros((N, m)), entropy=np.zeros(N), stats=np.zeros((N, 2)),
             top_idx=np.full((N, k), -1, np.int64), top_logp=np.full((N, k), -np.inf))
    for name in ("logp", "entropy", "stats", "top_logp"):
        r[name + "_err"] = np.zeros_like(r[name])
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for n in range(N):
            M = z[n].max()
            plain = np.isfinite(M)
            d = (z[n] - M) / tau if plain else np.full(V, np.nan)
            e = np.exp(d)
            S = e.sum() if plain else np.nan
            ls, p = np.log(S), e / S
            fin = np.where(np.isfinite(d), d, 0.0)
            some = p > 0
            H = ls - (p[some] * d[some]).sum() if plain else np.nan
            s_err = _softmax_error(fin, p, V) if plain else 0.0
            ls_err = s_err + 6 * EPS32 * abs(ls)
            r["stats"][n] = M, ls
            r["stats_err"][n] = 0.0, ls_err
            r["entropy"][n] = H
            Ed = (p * abs(fin)).sum()
            r["entropy_err"][n] = (ls_err + (p * abs(fin) * 4 * EPS32 * (2 + abs(fin))).sum() +
                                   Ed * (s_err + (_chain(V) + 8) * EPS32) + 4 * EPS32 * (abs(ls) + Ed))
            lp = d - ls
            lp_err = ls_err + 4 * EPS32 * (abs(fin) + abs(ls))
            used = (idx[n] >= 0) & (idx[n] < V)
            at = np.where(used, idx[n], 0)
            r["logp"][n] = np.where(used, lp[at], 0.0)
            r["logp_err"][n] = np.where(used, lp_err[at], 0.0)
            order = top_order(z[n])[:k]
            r["top_idx"][n, :len(order)] = order
            r["top_logp"][n, :len(order)] = lp[order]
            r["top_logp_err"][n, :len(order)] = lp_err[order]
    return r


def logprobs_grad(z, idx, tau, stats, entropy, d_logp, d_entropy, scale):
    """Gradient of the logits and its bound; stats, entropy: the floats given."""
    N, V = z.shape
    g, err = np.zeros((N, V)), np.zeros((N, V))
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for n in range(N):
            used = (idx[n] >= 0) & (idx[n] < V)
            dl = np.where(used, 0.0 if d_logp is None else d_logp[n], 0.0)
            dh = 0.0 if d_entropy is None else d_entropy[n]
            if not dl.any() and dh == 0:
                continue
            H = 0.0 if d_entropy is None else entropy[n]
            d, ls = (z[n] - stats[n, 0]) / tau, stats[n, 1]
            l = d - ls
            p = np.exp(l)
            fin = np.where(np.isfinite(l), l, 0.0)
            f = dl.sum() + dh * (fin + H)
            hit, mag = np.zeros(V), np.zeros(V)
            np.add.at(hit, idx[n][used], dl[used])
            np.add.at(mag, idx[n][used], abs(dl[used]))
            g[n] = scale / tau * (hit - np.where(p > 0, p * f, np.where(np.isnan(p), np.nan, 0.0)))
            # where p is below FP32's range it may be 0
            l_err = 4 * EPS32 * (abs(np.where(np.isfinite(d), d, 0)) + abs(ls) + 1)
            f_mag = abs(dl).sum() + abs(dh) * (abs(fin) + abs(H))
            err[n] = abs(scale / tau) * (p * (f_mag * (l_err + (len(dl) + 8) * EPS32) + abs(dh) * l_err) +
                                         len(dl) * EPS32 * mag + 3 * EPS32 * abs(hit - p * f) +
                                         2.0 ** -125 * f_mag)
    return g, err
