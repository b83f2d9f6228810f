"""Plain float64 definitions of the language-model operators, from the values of
the codes: rotary positions, attention with its gradients, the distillation
loss with its gradient.  Each row is computed from the keys it sees and nothing
else, so masked places cannot enter it.  The attention and distillation
functions also return bounds of the error a result in FP32 sums and IEEE-half
factors may have (see each).
"""
import numpy as np

EPS32 = 2.0 ** -24          # half a step of FP32, relative
EPS_HALF = 2.0 ** -11       # of IEEE half


def rotary(x, positions, freqs, interleaved=False, inverse=False, mscale=1.0):
    """x: T x H x D float64 values; returns the turned array."""
    n = len(freqs)
    a = np.asarray(positions, np.longdouble)[:, None] * np.asarray(freqs, np.longdouble)
    c, s = (f(a).astype(np.float64)[:, None] * mscale for f in (np.cos, np.sin))
    if inverse:
        s = -s
    i0 = 2 * np.arange(n) if interleaved else np.arange(n)
    i1 = i0 + 1 if interleaved else i0 + n
    y = x.copy()
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i1] * c + x[..., i0] * s
    return y


def _seen(i, nq, nk, causal):
    return max(0, min(nk, i + 1 + nk - nq)) if causal else nk


def attention(q, k, v, cu_q, cu_k, causal, sm_scale, e=None, o_given=None):
    """q: Tq x Hq x D, k, v: Tk x Hkv x D float64 values.  Returns a dict of o,
    lse (Hq x Tq) and, with e (the error of o), dq, dk, dv; and under "o_err",
    "lse_err", "dq_err", ... a bound of what FP32 arithmetic with IEEE-half
    factors may lose before the last rounding:

    * a score s_j: D exact products summed in FP32 in any order, one product
      by the scale, one subtraction: |s err| <= (D + 4) EPS32 c sum |q K_j|,
      plus EPS32 of |s_j| and of the maximum; both enter p as a relative error;
    * p: that, FP32 exp2 and sums ((nk + 8) EPS32), and EPS_HALF for the half
      factor (its absolute floor 2^-25 of the maximum is below that times p's
      share of 2^-14 and is added as nk 2^-39);
    * delta = <e, o>: o in FP16 (2^-10 relative) and its own error.
    """
    Tq, Hq, D = q.shape
    G = Hq // k.shape[1]
    r = dict(o=np.zeros_like(q), lse=np.full((Hq, Tq), -np.inf), o_err=np.zeros_like(q),
             lse_err=np.zeros((Hq, Tq)))
    if e is not None:
        for n, like in (("dq", q), ("dk", k), ("dv", v)):
            r[n], r[n + "_err"] = np.zeros_like(like), np.zeros_like(like)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for s in range(len(cu_q) - 1):
            nq, nk = cu_q[s + 1] - cu_q[s], cu_k[s + 1] - cu_k[s]
            for h in range(Hq):
                g = h // G
                for i in range(nq):
                    t, n = cu_q[s] + i, _seen(i, nq, nk, causal)
                    if n == 0:
                        continue
                    at = slice(cu_k[s], cu_k[s] + n)
                    K, V, Q = k[at, g], v[at, g], q[t, h]
                    x = sm_scale * (K @ Q)
                    m = x.max()
                    p = np.exp(x - m)
                    l = p.sum()
                    p /= l
                    r["lse"][h, t] = np.log(l) + m
                    o = r["o"][t, h] = p @ V
                    s_err = EPS32 * ((D + 4) * sm_scale * (np.abs(K) @ np.abs(Q)) + 2 * abs(x) +
                                     2 * abs(m))
                    p_err = s_err + s_err.max() + (n + 8) * EPS32
                    r["lse_err"][h, t] = s_err.max() + (n + 8) * EPS32 + 2 * EPS32 * abs(r["lse"][h, t])
                    half = p_err + 2 * EPS_HALF
                    r["o_err"][t, h] = (p * half + n * 2.0 ** -39) @ abs(V)
                    if e is None:
                        continue
                    E = e[t, h]
                    dP = V @ E
                    delta = E @ o
                    dS = p * (dP - delta) * sm_scale
                    d_err = abs(E) @ (2.0 ** -10 * abs(o) + r["o_err"][t, h]) + D * EPS32 * (
                        abs(E) @ abs(o))
                    t_err = D * EPS32 * (abs(V) @ abs(E)) + d_err
                    ds_err = abs(dS) * half + p * t_err * sm_scale + 2.0 ** -38 * sm_scale * (
                        abs(V) @ abs(E)).max()
                    r["dq"][t, h] = dS @ K
                    r["dq_err"][t, h] = ds_err @ abs(K) + n * EPS32 * (abs(dS) @ abs(K))
                    r["dk"][at, g] += dS[:, None] * Q
                    r["dk_err"][at, g] += (ds_err + nq * G * EPS32 * abs(dS))[:, None] * abs(Q)
                    r["dv"][at, g] += p[:, None] * E
                    r["dv_err"][at, g] += (p * (half + nq * G * EPS32) + 2.0 ** -39)[:, None] * abs(E)
    return r


def distill(z, idx, t, w, tau, grad_scale):
    """Loss (N) and gradient (N x V) of float64 logits, and bounds of their FP32
    errors: an exponent is one FMA from the exact logit (EPS32 of itself, plus
    the shared rounding of the maximum's, which cancels), exp2 and log2 a few
    EPS32, a sum of V terms (V / 64 + 64) EPS32 in any of the orders used."""
    N, V = z.shape
    loss, g = np.zeros(N), np.zeros((N, V))
    loss_err, g_err = np.zeros(N), np.zeros((N, V))
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        for n in range(N):
            use = (idx[n] >= 0) & (idx[n] < V)
            if w[n] == 0 or not use.any() or t[n][use].max() == -np.inf:
                continue
            y = t[n][use] / tau
            q = np.exp(y - y.max())
            q /= q.sum()
            x = z[n] / tau
            m = x.max()
            L = np.log(np.exp(x - m).sum())
            logp = x - m - L
            p = np.exp(logp)
            some = q > 0
            lq = np.log(q[some])
            loss[n] = w[n] * tau ** 2 * (q[some] * (lq - logp[idx[n][use][some]])).sum()
            g[n] = p
            np.subtract.at(g[n], idx[n][use], q)
            f = w[n] * tau * grad_scale
            g[n] *= f
            s_err = (V / 64 + 96) * EPS32
            x_err = 4 * EPS32 * (1 + np.abs(np.where(np.isfinite(x - m), x - m, 0)))
            y_err = 4 * EPS32 * (1 + abs(np.where(np.isfinite(y - y.max()), y - y.max(), 0)))
            q_err = q * (y_err + (len(q) + 8) * EPS32)
            lp = np.where(np.isfinite(logp), logp, 0)[idx[n][use][some]]
            loss_err[n] = w[n] * tau ** 2 * (
                q_err[some] * (abs(lq) + abs(lp) + 1) + q[some] * (
                    (y_err[some] + x_err[idx[n][use][some]]) + s_err +
                    8 * EPS32 * (abs(lq) + abs(lp)))).sum()
            g_err[n] = p * (x_err + s_err)
            np.add.at(g_err[n], idx[n][use], q_err)
            g_err[n] = abs(f) * (g_err[n] + 8 * EPS32 * (p + np.bincount(
                idx[n][use], q, minlength=V)))
    return loss, g, loss_err, g_err
