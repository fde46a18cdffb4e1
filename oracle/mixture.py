"""Mixture of generators: the choice of members, rows sorted by member and back, and the
members on rows of their own (test infrastructure).

Choices: p = softmax(scale * logits) of every row; ln p of given choices, the
entropy H = -sum p ln p, and the choices of the largest logits (of equal ones
the lowest first).  A logit of -infinity is masked.  The gradient follows
from d ln p_c / dz_v = [v = c] - p_v and dH / dz_v = -p_v (ln p_v + H).

Routing: item r * slots + k of row r goes to member[r][k]; items are sorted by
member, in their own order within one.  combine puts rows back with weights.

Pins (tests/test_oracle_mixture.py): softmax against scipy, gradients against
central differences and torch autograd, routing against a sort in pure Python.
"""
from __future__ import annotations

import numpy as np

from .generator import generator_backward, generator_forward


def log_probs(logits, scale=1.0):
    """ln p [n][V]: -infinity where masked."""
    z = scale * np.asarray(logits, dtype=np.float64)
    m = z.max(axis=1, keepdims=True)
    m = np.where(np.isneginf(m), 0.0, m)
    with np.errstate(divide="ignore", invalid="ignore"):
        lp = z - m - np.log(np.exp(z - m).sum(axis=1, keepdims=True))
    return np.where(np.isneginf(z), -np.inf, lp)


def choice_logprob(logits, choice=None, top=0, scale=1.0):
    lp = log_probs(logits, scale)
    n, V = lp.shape
    p = np.exp(lp)
    H = -np.where(p > 0, p * np.where(p > 0, lp, 0.0), 0.0).sum(axis=1)
    out = {"entropy": H + 0.0, "logp": None}
    if choice is not None:
        c = np.asarray(choice)
        on = (c >= 0) & (c < V)
        out["logp"] = np.where(on, lp[np.arange(n), np.where(on, c, 0)], 0.0)
    x = np.asarray(logits, dtype=np.float64)
    idx = np.argsort(-x, axis=1, kind="stable")[:, :top]
    tl = np.take_along_axis(lp, idx, axis=1)
    pad = top - idx.shape[1]
    idx = np.where(np.isneginf(tl), -1, idx)
    out["top_choice"] = np.pad(idx, ((0, 0), (0, pad)), constant_values=-1)
    out["top_logp"] = np.pad(tl, ((0, 0), (0, pad)), constant_values=-np.inf)
    return out


def choice_backward(logits, choice, d_logp=None, d_entropy=None, d_top=None, scale=1.0, with_terms=False):
    """dL/dlogits [n][V]; with_terms also the sum of the absolute terms of each."""
    lp = log_probs(logits, scale)
    n, V = lp.shape
    p = np.exp(lp)
    g = np.zeros((n, V))
    for r in range(n):
        if d_logp is not None and 0 <= choice[r] < V and np.isfinite(lp[r, choice[r]]):
            g[r, choice[r]] += d_logp[r]
    a = np.abs(g)
    if d_top is not None:
        f = choice_logprob(logits, None, d_top.shape[1], scale)
        for r in range(n):
            for k, c in enumerate(f["top_choice"][r]):
                if c >= 0:
                    g[r, c] += d_top[r, k]
                    a[r, c] += abs(d_top[r, k])
    dz = g - p * g.sum(axis=1, keepdims=True)
    terms = a + p * a.sum(axis=1, keepdims=True)
    if d_entropy is not None:
        H = choice_logprob(logits, None, 0, scale)["entropy"][:, None]
        lps = np.where(p > 0, lp, 0.0)
        dH = np.asarray(d_entropy, dtype=np.float64)[:, None]
        dz = dz - dH * np.where(p > 0, p * (lps + H), 0.0)
        terms = terms + np.abs(dH) * p * (np.abs(lps) + H)
    return (scale * dz, scale * terms) if with_terms else scale * dz


def route(member, n_members):
    member = np.asarray(member)
    n = member.size
    flat = member.reshape(-1)
    items = np.flatnonzero((flat >= 0) & (flat < n_members))
    order = items[np.argsort(flat[items], kind="stable")]
    place = np.full(n, -1)
    place[order] = np.arange(len(order))
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[items], minlength=n_members))])
    return {"offsets": offsets, "order": np.concatenate([order, np.full(n - len(order), -1)]), "place": place.reshape(member.shape)}


def combine(y, place, weight=None):
    """out [rows][width], and the sum of the absolute terms."""
    y = np.asarray(y, dtype=np.float64)
    rows, slots = place.shape
    out, terms = np.zeros((rows, y.shape[1])), np.zeros((rows, y.shape[1]))
    for k in range(slots):
        on = place[:, k] >= 0
        w = np.ones(rows) if weight is None else np.asarray(weight[:, k], dtype=np.float64)
        t = w[on, None] * y[place[on, k]]
        out[on] += t
        terms[on] += np.abs(t)
    return out, terms


def combine_backward(dout, y, place, weight=None):
    """dy (NaN at the positions of no item), dweight, and the sum of dweight's absolute terms."""
    dout, y = np.asarray(dout, dtype=np.float64), np.asarray(y, dtype=np.float64)
    rows, slots = place.shape
    dy = np.full((rows * slots, dout.shape[1]), np.nan)
    dw, terms = np.zeros((rows, slots)), np.zeros((rows, slots))
    for k in range(slots):
        on = place[:, k] >= 0
        at = place[on, k]
        w = np.ones(rows) if weight is None else np.asarray(weight[:, k], dtype=np.float64)
        dy[at] = w[on, None] * dout[on]
        dw[on, k] = (dout[on] * y[at]).sum(axis=1)
        terms[on, k] = np.abs(dout[on] * y[at]).sum(axis=1)
    return dy, dw, terms


def members_forward(W, b, x, offsets, slope=0.2):
    """theta [n][out]; rows of no member are NaN."""
    out = np.full((x.shape[0], W[-1].shape[1]), np.nan)
    for m in range(W[0].shape[0]):
        lo, hi = offsets[m], offsets[m + 1]
        if hi > lo:
            out[lo:hi] = generator_forward([w[m] for w in W], [v[m] for v in b], x[lo:hi], slope)
    return out


def members_backward(W, b, x, offsets, dL_dtheta, slope=0.2):
    """dW, db of every member, and dx (NaN for rows of no member)."""
    dW, db = [np.zeros(w.shape) for w in W], [np.zeros(v.shape) for v in b]
    dx = np.full(x.shape, np.nan)
    for m in range(W[0].shape[0]):
        lo, hi = offsets[m], offsets[m + 1]
        if hi <= lo:
            continue
        Wm, bm = [w[m].astype(np.float64) for w in W], [v[m].astype(np.float64) for v in b]
        gW, gb = generator_backward(Wm, bm, x[lo:hi], dL_dtheta[lo:hi], slope)
        for l in range(len(W)):
            dW[l][m], db[l][m] = gW[l], gb[l]
        f = generator_forward(Wm, bm, x[lo:hi], slope, return_all=True)
        g = np.asarray(dL_dtheta[lo:hi], dtype=np.float64) / (1.0 + np.exp(-f["pres"][-1]))
        for l in range(len(W) - 1, -1, -1):
            g = g @ Wm[l]
            if l:
                g = g * np.where(f["pres"][l - 1] > 0, 1.0, slope)
        dx[lo:hi] = g
    return dW, db, dx
