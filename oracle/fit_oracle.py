"""Oracle of the training side (Sec. 4.3): sorted indices, router losses, gated lookup, and their gradients, numpy float64.

TEST INFRASTRUCTURE ONLY.  Everything is written out as its definition, one group at a time:

    M = x W^T + b,  p = softmax(M) by row,  lse = log sum exp M
    mean_j = average of p_ij over the positions that take part,  balance = sum_j mean_j log(mean_j m)
    peak = average of -log sigmoid(M[i, I_i])
    out_i = (user_i | sigmoid(s_i) pool[I_i])

A position takes part in a group if its index lies in [0, m).  Inputs may be bfloat16 bit patterns (uint16), widened
exactly.
"""
from __future__ import annotations

import numpy as np


def f64(a):
    if a is None:
        return None
    if a.dtype == np.uint16:
        return (a.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)
    return a.astype(np.float64)


def sigmoid(x):
    return np.exp(np.minimum(x, 0)) / (1 + np.exp(-np.abs(x)))


def takes_part(idx, m):
    return (idx >= 0) & (idx < m)


def sort_indices(idx, m):
    """order [G][n], offset [G][m + 1]"""
    key = np.where(takes_part(idx, m), idx, m).T
    order = np.argsort(key, axis=1, kind="stable").astype(np.int32)
    offset = np.stack([np.searchsorted(np.sort(k), np.arange(m + 1), side="left") for k in key]).astype(np.int32)
    return order, offset


def _softmax(M):
    """p and lse by row; a row of -inf has no weight anywhere."""
    top = M.max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.where(np.isneginf(top), 0.0, np.exp(M - top))
        total = e.sum(1, keepdims=True)
        lse = np.where(total > 0, np.log(total) + top, -np.inf)[:, 0]
    return np.divide(e, total, out=np.zeros_like(e), where=total > 0), lse


def scores(x, W, bias, g):
    with np.errstate(invalid="ignore"):
        M = f64(x) @ f64(W[g]).T
    return M if bias is None else M + f64(bias[g])


def taken_out(bias, g):
    """What to add to the scores: -inf for an entry whose bias is -2^20 or less."""
    return 0.0 if bias is None else np.where(f64(bias[g]) <= -2.0 ** 20, -np.inf, 0.0)


def route_loss(x, W, bias, idx):
    n, (G, m, _) = x.shape[0], W.shape
    loss, lse, score, mean = np.zeros((G, 2)), np.zeros((n, G)), np.zeros((n, G)), np.zeros((G, m))
    for g in range(G):
        rows = np.nonzero(takes_part(idx[:, g], m))[0]
        if len(rows) == 0:
            continue
        M = scores(x[rows], W, bias, g)
        p, lse[rows, g] = _softmax(M + taken_out(bias, g))
        score[rows, g] = M[np.arange(len(rows)), idx[rows, g]]
        mean[g] = p.mean(0)
        used = mean[g] > 0
        loss[g, 0] = (mean[g][used] * np.log(mean[g][used] * m)).sum()
        s = score[rows, g]
        loss[g, 1] = (np.log1p(np.exp(-np.abs(s))) + np.maximum(-s, 0)).mean()
    return loss, lse, score, mean


def route_loss_grad(x, W, bias, idx, mean, w_balance, w_peak, d_score=None, lse=None):
    """dx, dW, dbias, and for each the sum of the absolute values of its terms: (T's, what T's own error scales with).
    lse: the given one [n][G] instead of the one of the scores."""
    (n, d), (G, m, _) = x.shape, W.shape
    dx, dW, db = np.zeros((n, d)), np.zeros((G, m, d)), np.zeros((G, m))
    size = {k: [np.zeros_like(v), np.zeros_like(v), np.zeros_like(v)] for k, v in dict(dx=dx, dW=dW, db=db).items()}
    for g in range(G):
        rows = np.nonzero(takes_part(idx[:, g], m))[0]
        if len(rows) == 0:
            continue
        X, Wg = f64(x[rows]), f64(W[g])
        M = scores(x[rows], W, bias, g)
        S = M + taken_out(bias, g)
        p, own = _softmax(S)
        if lse is not None:
            with np.errstate(invalid="ignore"):
                p = np.where(np.isneginf(S), 0.0, np.exp(S - lse[rows, g][:, None])) if len(rows) else p
        u = mean[g] * m
        h = np.where(u > 0, np.log(np.where(u > 0, u, 1)), 0.0) * w_balance / len(rows)
        r = p @ h
        T = p * (h[None] - r[:, None])
        A = p * (np.abs(h)[None] + (p @ np.abs(h))[:, None])
        ds = -w_peak / len(rows) * sigmoid(-M[np.arange(len(rows)), idx[rows, g]])
        if d_score is not None:
            ds = ds + d_score[rows, g]
        picked = np.zeros_like(T)
        picked[np.arange(len(rows)), idx[rows, g]] = ds
        dM = T + picked
        dx[rows] += dM @ Wg
        dW[g], db[g] = dM.T @ X, dM.sum(0)
        for i, t in enumerate((np.abs(T), A, np.abs(picked))):
            size["dx"][i][rows] += t @ np.abs(Wg)
            size["dW"][i][g], size["db"][i][g] = t.T @ np.abs(X), t.sum(0)
    return dx, dW, db, size


def gather(pool, idx, user, score=None):
    P, (n, G) = f64(pool), idx.shape
    m = P.shape[1]
    rows = np.zeros((n, G, P.shape[2]))
    for g in range(G):
        k = takes_part(idx[:, g], m)
        rows[k, g] = P[g][idx[k, g]] * (1.0 if score is None else sigmoid(f64(score[k, g]))[:, None])
    return rows if user is None else np.concatenate([f64(user), rows], 2)


def gather_grad(pool, idx, score, d_out):
    """d_pool, d_user, d_score, and the sums of the absolute values of the terms of d_pool and d_score"""
    P, dO = f64(pool), f64(d_out)
    (G, m, ds), n = P.shape, idx.shape[0]
    du = dO.shape[2] - ds
    d_pool, d_score = np.zeros((G, m, ds)), np.zeros((n, G))
    a_pool, a_score = np.zeros_like(d_pool), np.zeros_like(d_score)
    for g in range(G):
        k = np.nonzero(takes_part(idx[:, g], m))[0]
        gate = np.ones(len(k)) if score is None else sigmoid(f64(score[k, g]))
        t = gate[:, None] * dO[k, g, du:]
        np.add.at(d_pool[g], idx[k, g], t)
        np.add.at(a_pool[g], idx[k, g], np.abs(t))
        if score is not None:
            c = gate * sigmoid(-f64(score[k, g]))
            d_score[k, g] = c * (P[g][idx[k, g]] * dO[k, g, du:]).sum(1)
            a_score[k, g] = c * np.abs(P[g][idx[k, g]] * dO[k, g, du:]).sum(1)
    return d_pool, dO[:, :, :du], d_score, a_pool, a_score
