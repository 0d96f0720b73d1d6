"""The operators over a whole item table in 64 bits, from their definitions, with bounds on what a computation
with 32-bit sums may be off.

Bounds, per value, u = 2^-24 half a step of fp32:
  * a score is off by at most (K + 16) 2 u A_ij, A_ij = sum_k |x_k w_k|: K additions, the products' planes of
    22 bits (three products dropped or rounded at 2^-22 each make 12 u), and the scaling;
  * a weight exp(s - lse) is off by that of s and of lse, and 2^-20 of the exponential and of its two
    planes of 22 bits; a sum of M of them adds (M + 64) u;
  * bf16 tables: the item gradients' weights g (V p - y) are held in one fp16 number each, off by half a step,
    2^-11 of themselves (2^-25 of the largest share below 2^-14 of it, within the 2^-34 of the shares' sums below);
  * what is rounded to the tables' type adds half a step of it, and half its smallest step.
"""
import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def lists_of(item, row_ptr, n, M):
    """Entries in range, as (row, entry) pairs."""
    item = np.asarray(item.cpu())
    if row_ptr is None:
        rows = np.arange(n)
        at = np.arange(n)
    else:
        ptr = np.asarray(row_ptr.cpu())
        rows = np.repeat(np.arange(n), np.diff(ptr))
        at = np.arange(ptr[0], ptr[-1])
    keep = (item[at] >= 0) & (item[at] < M)
    return rows[keep], at[keep], item[at[keep]]


def dense_loss(x, w, y, extra, live, weight, tau, halves=False):
    """Losses, log-sum-exps, gradients of weighted rows with target weights y (n x M), and their bounds."""
    n, K = x.shape
    M = w.shape[0]
    live = live & (weight != 0)
    x = np.where(live[:, None], x, 0.0)
    y = np.where(live[:, None], y, 0.0)
    s = x @ w.T / tau
    a = np.abs(x) @ np.abs(w).T / tau
    top = s.max(1, keepdims=True)
    lse = np.log(np.exp(s - top).sum(1)) + top[:, 0]
    p = np.exp(s - lse[:, None])
    V, Va = y.sum(1), np.abs(y).sum(1)
    gain = tau * tau
    loss = np.where(live, gain * (extra + V * lse - (y * s).sum(1)), 0.0)
    g = np.where(live, weight * tau, 0.0)
    dS = g[:, None] * (V[:, None] * p - y)
    dX, dW = dS @ w, dS.T @ x
    # bounds
    least = 2.0 ** -36 * np.abs(x).max(initial=0.0) * np.abs(w).max() * K / tau  # numbers far below their table's largest
    es = (K + 16) * 2 * U * a + least
    elog = es.max(1) + (M + 64) * U + 4 * U * np.abs(lse)
    ey = (K + 16) * 2 * U * a
    cnt = (y != 0).sum(1)
    eloss = gain * ((np.abs(y) * (ey + elog[:, None] + 8 * U * (np.abs(s) + np.abs(lse)[:, None]))).sum(1)
                    + (cnt + 16) * 2 * U * (np.abs(extra) + (np.abs(y) * np.abs(lse[:, None] - s)).sum(1))
                    + 64 * U * Va * (1 + np.abs(lse)))
    ep = es + elog[:, None] + 2.0 ** -20 + (M + n + 64) * U
    big = np.abs(g * V)[:, None] * p * ep
    exact = np.abs(g)[:, None] * np.abs(y) * (max(n, 1) + M + 16) * U
    eX = (big + exact) @ np.abs(w) + 2.0 ** -34 * np.abs(g * V)[:, None] * np.abs(w).max()
    eW = (big + exact).T @ np.abs(x) + 2.0 ** -34 * np.abs(g * V).max(initial=0.0) * np.abs(x).max(initial=0.0)
    if halves:
        eW = eW + 2.0 ** -11 * (np.abs(dS) + big + exact).T @ np.abs(x) + 2.0 ** -32 * np.abs(g).max(initial=0.0) * Va.max(initial=0.0) * np.abs(x).sum(0)
    return (loss, lse, dX, dW), (eloss, elog, eX, eW)


def xent(X, W, item, row_ptr=None, value=None, weight=None):
    x, w = f64(X), f64(W)
    n, M = x.shape[0], w.shape[0]
    rows, at, items = lists_of(item, row_ptr, n, M)
    v = np.ones(len(at)) if value is None else f64(value)[at]
    y = np.zeros((n, M))
    np.add.at(y, (rows, items), v)
    live = np.zeros(n, bool)
    live[rows] = True
    wt = np.ones(n) if weight is None else f64(weight)
    return dense_loss(x, w, y, np.zeros(n), live, wt, 1.0, X.dtype == torch.bfloat16)


def distill(X, W, item, score, tau, tlse=None, weight=None):
    x, w, t = f64(X), f64(W), f64(score) / tau
    n, M = x.shape[0], w.shape[0]
    it = np.asarray(item.cpu())
    here = (it >= 0) & (it < M)
    t = np.where(here, t, -np.inf)
    here &= t > -np.inf
    live = here.any(1)
    if tlse is None:
        top = np.where(live, t.max(1), 0.0)[:, None]
        with np.errstate(divide="ignore"):
            z = np.log(np.exp(t - top).sum(1, keepdims=True)) + top
    else:
        z = f64(tlse)[:, None]
    with np.errstate(invalid="ignore"):
        lq = np.where(here, t - np.where(live[:, None], z, 0.0), -np.inf)
    q = np.exp(lq)
    extra = np.where(q > 0, q * np.where(here, lq, 0.0), 0.0).sum(1)
    y = np.zeros((n, M))
    r, c = np.nonzero(here)
    np.add.at(y, (r, it[r, c]), q[r, c])
    wt = np.ones(n) if weight is None else f64(weight)
    vals, errs = dense_loss(x, w, y, extra, live, wt, tau, X.dtype == torch.bfloat16)
    # q itself comes from fp32: each is off by eq of itself, t and z up to 4 u of themselves
    live = live & (wt != 0)
    eq = 2.0 ** -20 + 8 * U * (np.abs(np.where(here, t, 0.0)).max(1) + np.abs(np.where(live, z[:, 0], 0.0)))
    loss, lse, dX, dW = vals
    s = np.where(live[:, None], x, 0.0) @ w.T / tau
    gap = (y * (1 + np.abs(lse[:, None] - s))).sum(1) + (q * np.where(here, np.abs(lq) + 1, 0.0)).sum(1)
    g = np.abs(np.where(live, wt * tau, 0.0))
    p = np.exp(s - lse[:, None])
    off = g[:, None] * eq[:, None] * (y.sum(1, keepdims=True) * p + y)
    return vals, (errs[0] + tau * tau * eq * gap, errs[1], errs[2] + off @ np.abs(w),
                  errs[3] + off.T @ np.abs(np.where(live[:, None], x, 0.0)))


def top(X, W, k, row_ptr=None, item=None):
    s = f64(X) @ f64(W).T
    n, M = s.shape
    out = np.ones((n, M), bool)
    if row_ptr is not None:
        rows, _, items = lists_of(item, row_ptr, n, M)
        out[rows, items] = False
    best = np.full((n, k), -1, np.int32)
    score = np.full((n, k), -np.inf)
    for i in range(n):
        at = np.nonzero(out[i])[0]
        v = s[i, at]
        order = np.lexsort((at, np.where(np.isnan(v), -np.inf, -v)))[:k]
        best[i, : len(order)] = at[order]
        score[i, : len(order)] = v[order]
    return best, score.astype(np.float32)


def near(got, want, bound, dtype=torch.float32):
    """The largest |got - want| over its bound (at most 1: fine)."""
    got = f64(got)
    assert got.shape == want.shape, (got.shape, want.shape)
    if got.size == 0:
        return 0.0
    assert np.isfinite(got).all(), "not finite"
    room = bound + (HALF[dtype] * (np.abs(want) + bound)) * 1.01 + LEAST[dtype]
    return float((np.abs(got - want) / room).max())
