"""fp64 oracle of the calls beside the scoring path: LM-head loss and its gradients, attention of
drafted tokens over a cache, eviction.  Plain definitions, sequence by sequence and head by head;
shares no code with the HIP path.

Every ``*_bounds`` value returned next to a result says how far a computation in 32 bits, with the
roundings the library documents, can be from it at most; u = 2^-24, gamma_n = n u / (1 - n u).
"""
from __future__ import annotations

import numpy as np

from .estp_oracle import widen

U = 2.0 ** -24


def gamma(n) -> float:
    return n * U / (1.0 - n * U)


def _rounding(dtype: str) -> float:
    """Largest relative error of rounding to the type."""
    return 2.0 ** -8 if dtype == "bf16" else U


def _two_parts(dtype: str) -> float:
    """Largest relative error of a number as the sum of two of the type (bf16), or as one (fp32)."""
    return 2.0 ** -16 if dtype == "bf16" else U


def token_loss(X, W, targets):
    """(loss [n], lse [n]): lse_i = log sum_v exp(W_v . x_i), loss_i = lse_i - W_t . x_i; 0 where the
    target lies outside [0, V)."""
    X, W, t = widen(X), widen(W), np.asarray(targets)
    z = X @ W.T
    m = z.max(axis=1)
    lse = m + np.log(np.exp(z - m[:, None]).sum(axis=1))
    live = (t >= 0) & (t < W.shape[0])
    loss = np.zeros(len(X))
    rows = np.flatnonzero(live)
    loss[rows] = lse[rows] - z[rows, t[rows]]
    return loss, lse


def logit_bound(X, W):
    """Per row: any fp32 summation of the d exact (bf16) or once-rounded (fp32) products of a logit is within
    gamma_{d+1} sum |w x| of it."""
    X, W = np.abs(widen(X)), np.abs(widen(W))
    return gamma(X.shape[1] + 1) * (X @ W.T).max(axis=1)


def lse_bound(X, W, lse):
    """The log-sum-exp moves by at most the largest logit error; the running sums and rescalings of up to
    ceil(V / 256) + 32 tiles and partial states add, each, one rounding of the reference (a number of the size
    of lse log2 e) and one of the sum, and the exponentials two units: relative to 1 or to |lse|."""
    n = (W.shape[0] + 255) // 256 + 32
    return logit_bound(X, W) + n * 4 * U * (1.0 + np.abs(lse))


def token_loss_grads(X, W, targets, grad, dtype: str, lse=None):
    """(dX, dW, bound_dX, bound_dW) of sum_i grad_i loss_i.  Bounds: G rounded to the type once (in two parts of up
    to 64 tokens), its p_iv off by the relative error of its exponent and of exp2 (2 units), fp32 sums of V or n terms
    a part, one rounding at the end."""
    dX_in, W64, t = widen(X), widen(W), np.asarray(targets)
    n, d = dX_in.shape
    V = W64.shape[0]
    live = np.flatnonzero((t >= 0) & (t < V))
    dX, bX = np.zeros((n, d)), np.zeros((n, d))
    x, g = dX_in[live], np.asarray(grad, dtype=np.float64)[live]
    z = x @ W64.T
    m = z.max(axis=1, keepdims=True)
    l64 = m[:, 0] + np.log(np.exp(z - m).sum(axis=1))
    P = np.exp(z - l64[:, None])
    G = P.copy()
    G[np.arange(len(live)), t[live]] -= 1.0
    G *= g[:, None]
    r = _rounding(dtype)
    rg = _two_parts(dtype) if n <= 64 else r
    eps = np.zeros(len(live))
    if len(live):
        # exponent: the logit, the given lse, and the roundings of (z - lse) log2 e
        eps = 1.01 * (logit_bound(x, W64) + lse_bound(x, W64, l64) + 8 * U * (np.abs(z).max(axis=1) + np.abs(l64)))
        eps += 4 * U
    dG = np.abs(G) * rg * 1.01 + np.abs(g)[:, None] * (P * eps[:, None] + 2 * U * P + 2 * U)* (1.0 + r)
    dX[live] = G @ W64
    aW, ax = np.abs(W64), np.abs(x)
    bX[live] = (dG + gamma(2 * V + 8) * np.abs(G)) @ aW * (1.0 + r) + r * np.abs(dX[live])
    dW = G.T @ x
    bW = (dG + gamma(2 * len(live) + 8) * np.abs(G)).T @ ax * (1.0 + r) + r * np.abs(dW)
    return dX, dW, bX, bW


def tree_attention(Q, K, V, lens, cu_q, tree_mask=None, scale=None, dtype: str = "f32", row_weight=None):
    """Q [n_q, Hq, dh], K, V [B, Hkv, cap, dh]; tree_mask: Python ints or None (a chain).

    Returns a dict: O, lse, got [B, Hkv, cap] (the weight each slot receives, rows counting row_weight), and the
    bounds O_bound, lse_bound, got_bound."""
    Q, K, V = widen(Q), widen(K), widen(V)
    n_q, Hq, dh = Q.shape
    B, Hkv, cap = K.shape[:3]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(dh) if scale is None else scale
    r = _rounding(dtype)
    out = {"O": np.zeros((n_q, Hq, dh)), "lse": np.full((Hq, n_q), -np.inf), "got": np.zeros((B, Hkv, cap))}
    out.update({k + "_bound": np.zeros_like(v) for k, v in out.items()})
    for b in range(B):
        T = int(cu_q[b + 1] - cu_q[b])
        n = int(lens[b])
        for t in range(T):
            i = int(cu_q[b]) + t
            mask = (2 << t) - 1 if tree_mask is None else int(tree_mask[i])
            sees = [j for j in range(T) if mask >> j & 1]
            keys = np.concatenate([np.arange(n), n + np.array(sees, dtype=np.int64)]).astype(np.int64)
            if len(keys) == 0:
                continue
            w = 1.0 if row_weight is None else float(row_weight[i])
            for h in range(Hq):
                k, v, q = K[b, h // G][keys], V[b, h // G][keys], Q[i, h]
                s = scale * (k @ q)
                # fp32 scores: dh products and sums, the scale in base 2 (3 roundings)
                ds = gamma(dh + 6) * abs(scale) * (np.abs(k) @ np.abs(q)) + 4 * U * np.abs(s)
                m = s.max()
                e = np.exp(s - m)
                lse = m + np.log(e.sum())
                p = np.exp(s - lse)
                # running maximum and sum over tiles and ranges: a few units each
                dl = float((p * ds).sum()) * 1.01 + 4 * U * (np.abs(m) + np.abs(lse) + 1.0) + gamma(len(keys) + 64)
                out["O"][i, h] = p @ v
                out["lse"][h, i] = lse
                out["lse_bound"][h, i] = dl
                rel = 1.01 * (ds + dl + 4 * U * (np.abs(s) + abs(lse) + 1.0))
                # weights in two parts, fp32 sums, one rounding of the result
                dp = p * (rel + 1.01 * _two_parts(dtype) + gamma(2 * len(keys) + 64))
                out["O_bound"][i, h] = (dp @ np.abs(v)) * (1 + r) + r * np.abs(out["O"][i, h])
                if w != 0.0:
                    out["got"][b, h // G, keys] += w * p
                    out["got_bound"][b, h // G, keys] += abs(w) * p * (rel + gamma(2 * T * G + 8))
    return out


def cache_evict(acc, pos, lens, seen, keep: int, recent: int = 0, sink: int = 0):
    """(idx [B, Hkv, keep], lens_out [B]): guarded slots first, then the largest weights (NaN lowest), the lowest
    slot among equals; kept slots at or past ``keep`` fill the holes below it in ascending order."""
    acc, pos = np.asarray(acc), np.asarray(pos)
    B, Hkv, _ = acc.shape
    idx = np.full((B, Hkv, keep), -1, dtype=np.int64)
    for b in range(B):
        n = int(lens[b])
        for g in range(Hkv):
            def rank(i):
                w = float(acc[b, g, i])
                guarded = pos[b, g, i] < sink or pos[b, g, i] >= int(seen[b]) - recent
                return (not guarded, w != w, 0.0 if w != w else -w, i)
            kept = set(sorted(range(n), key=rank)[:keep])
            holes = [i for i in range(min(n, keep)) if i not in kept]
            late = sorted(i for i in kept if i >= keep)
            for i in kept:
                if i < keep:
                    idx[b, g, i] = i
            for dst, src in zip(holes, late):
                idx[b, g, dst] = src
    return idx, np.minimum(np.asarray(lens), keep)


def evicted(a, idx, lens, fill):
    """What ``acc`` or ``pos`` [B, Hkv, cap] become: kept values first, ``fill`` up to the old length."""
    out = np.array(a)
    B, Hkv, keep = idx.shape
    for b in range(B):
        for g in range(Hkv):
            m = idx[b, g][idx[b, g] >= 0]
            out[b, g, :len(m)] = a[b, g, m]
            out[b, g, len(m):int(lens[b])] = fill
    return out
