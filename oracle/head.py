"""fp64 oracle of the calls that give log-probabilities over the LM head: alternatives and entropy of a token's
distribution, distillation from a teacher's top tokens and its gradients.  Plain definitions, row by row; shares no code
with the HIP path.

Every ``*_bound`` says how far a computation in 32 bits, with the roundings the library documents, can be from the value
next to it at most; u = 2^-24, gamma_n = n u / (1 - n u).
"""
from __future__ import annotations

import numpy as np

from .estp_oracle import widen
from .operators import U, _rounding, _two_parts, gamma, logit_bound, lse_bound


def _scaled_bound(X, W, s, temperature):
    """Per row: a scaled logit is off by its logit's error, by the two roundings of a product with the rounded inverse
    of the temperature, and by as many again of its base-2 form."""
    return logit_bound(X, W) / temperature + 4 * U * np.abs(s).max(axis=1)


def _scaled(X, W, temperature):
    X, W = widen(X), widen(W)
    s = X @ W.T / temperature
    m = s.max(axis=1)
    return s, m + np.log(np.exp(s - m[:, None]).sum(axis=1))


def _lse_bound(X, W, s, lse, temperature):
    return _scaled_bound(X, W, s, temperature) + lse_bound(X, W, lse) - logit_bound(X, W)


def token_logprobs(X, W, targets, k, temperature=1.0):
    """A dict: logprob, lse, H, top_id (stable descending order of the exact logits), top_logprob, their bounds, and
    `margin`: logits that are further apart than this keep their order."""
    s, lse = _scaled(X, W, temperature)
    n, V = s.shape
    t = np.full(n, -1) if targets is None else np.asarray(targets)
    live = np.flatnonzero((t >= 0) & (t < V))
    logprob = np.zeros(n)
    logprob[live] = s[live, t[live]] - lse[live]
    logp = s - lse[:, None]
    p = np.exp(logp)
    H = -(p * logp).sum(axis=1)
    top = np.argsort(-s, axis=1, kind="stable")[:, :k]
    bl = _lse_bound(X, W, s, lse, temperature)
    ds = _scaled_bound(X, W, s, temperature)
    out = {"s": s, "lse": lse, "logprob": logprob, "H": H, "top_id": top, "top_logprob": np.take_along_axis(logp, top, 1)}
    out["lse_bound"] = bl
    # a scaled logit's error, that of lse and the rounding of their difference
    out["logprob_bound"] = ds + bl + U * (np.abs(lse) + np.abs(s).max(axis=1))
    # dH / ds_v = -p_v (log p_v + H): at most 2 H in all.  Sums of p (s - ref), whose absolute values add up to 2 H at
    # most (ref lies between the largest logit and lse, which is H above it at most), over the chains that lse_bound
    # counts, and roundings of the rebased references
    chains = (V + 255) // 256 + 32
    out["H_bound"] = 2 * (H + 1) * ds + chains * 8 * U * (1 + H + np.abs(lse))
    out["margin"] = 2 * logit_bound(X, W) / temperature
    return out


def _teacher(ids, logp, V, renormalise):
    """(held [n, K], p, log p, relative error of p in 32 bits), 0, -inf and 0 of entries that are not held."""
    ids, lp = np.asarray(ids), np.asarray(logp, dtype=np.float64)
    held = (ids >= 0) & (ids < V)
    lp = np.where(held, lp, -np.inf)
    err = np.where(np.isfinite(lp), np.abs(lp), 0.0)
    if renormalise:
        m = np.maximum(lp.max(axis=1, keepdims=True), -1e300)
        total = np.exp(lp - m).sum(axis=1, keepdims=True)
        lp = np.where(total > 0, lp - m - np.log(np.where(total > 0, total, 1.0)), -np.inf)
        err = np.where(np.isfinite(lp), np.abs(lp), 0.0) + err + np.abs(m) * (m > -1e300)
    p = np.exp(lp)
    # exponents rounded three times, exp2 and log2 two units each, a sum of K
    return held, p, lp, 4 * U * err + (12 + gamma(ids.shape[1]) / U) * U


def distill(X, W, ids, logp, temperature=1.0, renormalise=True, grad=None, dtype="f32"):
    """A dict: loss, lse, logq, with `grad` also dX and dW, and their bounds."""
    s, lse = _scaled(X, W, temperature)
    n, V = s.shape
    ids = np.asarray(ids)
    K = ids.shape[1]
    held, p, lp, ep = _teacher(ids, logp, V, renormalise)
    at = np.where(held, ids, 0)
    logq = np.where(held, np.take_along_axis(s, at, 1) - lse[:, None], 0.0)
    with np.errstate(invalid="ignore"):
        term = np.where(p > 0, p * (lp - logq), 0.0)
        gap = np.where(p > 0, np.abs(lp) + np.abs(logq), 0.0)
    ds, bl = _scaled_bound(X, W, s, temperature), _lse_bound(X, W, s, lse, temperature)
    bq = ds + bl + 2 * U * (np.abs(lse) + np.abs(s).max(axis=1))
    out = {"loss": term.sum(axis=1), "lse": lse, "logq": logq, "lse_bound": bl,
           "logq_bound": bq[:, None] * np.ones((1, K))}
    out["loss_bound"] = (p * (ep * (1 + gap) + bq[:, None] + 2 * U * gap) + gamma(K + 4) * p * gap).sum(axis=1)
    if grad is None:
        return out
    X64, W64 = widen(X), widen(W)
    g = np.asarray(grad, dtype=np.float64) / temperature
    live = np.flatnonzero((np.where(held, np.asarray(logp, dtype=np.float64), -np.inf) > -np.inf).any(axis=1))
    x, gl = X64[live], g[live]
    P = p[live].sum(axis=1)
    q = np.exp(s[live] - lse[live, None])
    target, e_target = np.zeros_like(q), np.zeros_like(q)
    for j, i in enumerate(live):
        np.add.at(target[j], at[i][held[i]], p[i][held[i]])
        np.add.at(e_target[j], at[i][held[i]], (p[i] * ep[i])[held[i]])
    G = gl[:, None] * (P[:, None] * q - target)
    r = _rounding(dtype)
    rg = _two_parts(dtype) if n <= 64 else r
    # relative error of a weight: of its exponent (logit, lse, their roundings and those of the change of base) and
    # exp2; of the mass: that of its parts and their sum
    eq = 1.01 * (bq[live] + 8 * U * (np.abs(s[live]).max(axis=1) + np.abs(lse[live]))) + 4 * U
    eP = ((p * ep)[live].sum(axis=1) + gamma(K + 4) * P)[:, None]
    dG = np.abs(G) * rg * 1.01 + np.abs(gl)[:, None] * (P[:, None] * q * (eq[:, None] + 6 * U) + q * eP + e_target
                                                        + (6 * U + gamma(K)) * target) * (1.0 + r)
    dX, bX = np.zeros_like(X64), np.zeros_like(X64)
    dX[live] = G @ W64
    bX[live] = (dG + gamma(2 * V + 8) * np.abs(G)) @ np.abs(W64) * (1.0 + r) + r * np.abs(dX[live])
    dW = G.T @ x
    bW = (dG + gamma(2 * len(live) + 8) * np.abs(G)).T @ np.abs(x) * (1.0 + r) + r * np.abs(dW)
    out.update(dX=dX, dW=dW, dX_bound=bX, dW_bound=bW)
    return out
