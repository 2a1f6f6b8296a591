"""Windowed attention with sinks in 64 bits, from its definition, with the bound that the roundings of the bf16 path leave.

A rounding is off by at most half a step: U = 2^-8 of the value for bf16.  The path rounds, besides its results: the
probabilities P before they meet V and dO, dS before it meets K and Q (in dK from the rounded P), and takes Delta from the
rounded o.  A few 1e-4 of the sums of magnitudes cover what fp32 sums, products and exponentials add."""
import numpy as np

U, F32 = 2.0 ** -8, 2e-4


def allowed(n, window, sinks):
    i, j = np.arange(n)[:, None], np.arange(n)[None]
    return (j <= i) & ((i - j < window) | (j < sinks))


def window_attention(q, k, v, cu, window, sinks, scale, d_o=None, u=U):
    """q [T, nq, d], k, v [T, nkv, d] -> {name: (value, bound)} of o, lse [nq, T] and, with d_o, dq, dk, dv"""
    T, nq, d = q.shape
    g = nq // k.shape[1]
    out = {n: (np.zeros_like(t), np.zeros_like(t)) for n, t in (("o", q), ("dq", q), ("dk", k), ("dv", v))}
    out["lse"] = np.zeros((nq, T)), np.zeros((nq, T))
    for a, b in zip(cu[:-1], cu[1:]):
        m = allowed(b - a, window, sinks)
        for h in range(nq):
            Q, K, V = q[a:b, h], k[a:b, h // g], v[a:b, h // g]
            S = np.where(m, scale * (Q @ K.T), -np.inf)
            top = S.max(1, keepdims=True)
            e = np.exp(S - top)
            P = e / e.sum(1, keepdims=True)
            o, mag = P @ V, P @ np.abs(V)
            o_err = u * (mag + np.abs(o)) + F32 * mag
            out["o"][0][a:b, h], out["o"][1][a:b, h] = o, o_err
            out["lse"][0][h, a:b] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
            out["lse"][1][h, a:b] = 1e-5 * (1 + scale * (np.abs(Q) @ np.abs(K).T).max(1))
            if d_o is None:
                continue
            G = d_o[a:b, h]
            dP = G @ V.T
            dS = P * (dP - (G * o).sum(1, keepdims=True))
            delta_err = (np.abs(G) * o_err).sum(1, keepdims=True)
            # of a value of dS: two roundings, what Delta is off by, and of fp32 a share of the terms that cancel in it
            dS_err = 2 * u * np.abs(dS) + P * delta_err + F32 * P * (np.abs(G) @ np.abs(V).T + np.abs(G * o).sum(1, keepdims=True))
            for n, rows, val, err in (("dq", h, scale * dS @ K, scale * dS_err @ np.abs(K)),
                                      ("dk", h // g, scale * dS.T @ Q, scale * dS_err.T @ np.abs(Q)),
                                      ("dv", h // g, P.T @ G, (u + F32) * P.T @ np.abs(G))):
                out[n][0][a:b, rows] += val
                out[n][1][a:b, rows] += err
    for n in ("dq", "dk", "dv"):
        out[n][1][...] += u * np.abs(out[n][0]) + 1e-30
    return out
