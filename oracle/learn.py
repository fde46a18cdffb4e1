"""Training without a differentiable pipeline, in float64 (test infrastructure).

The policy is the sampler's density: an event x drawn at the row
(a_1, b_1, ..., a_d, b_d) has, for independent Kumaraswamy coordinates,

  l(x) = sum_j ln a_j + ln b_j + (a_j - 1) ln x_j + (b_j - 1) ln(1 - x_j^a_j).

policy_loss is the clipped surrogate of Schulman et al. (2017), eq. 7, with the
KL estimate exp(r) - 1 - r, r = l_ref - l_theta; preference_loss the logistic
loss of paired log ratios (Rafailov et al. 2023, eq. 7) with label smoothing,
over event sets; group_advantage centres and scales rewards within a row.

orthogonalise and muon_step: at the end of the file.

Pins (tests/test_oracle_learn.py): the density integrates to one and is the
derivative of the sampler's CDF, its gradient and both losses' gradients by
finite differences, closed values where nothing has moved, and the
orthogonalisation against its matrix products.
"""
from __future__ import annotations

import numpy as np

X_LO, X_HI = 2.0 ** -126, 1.0 - 2.0 ** -24


def event_logp(theta, x):
    """l [n], dl/dtheta [n][2d] and the absolute values of the latter's terms, summed, of events x [n][d]
    at rows theta [n][2d] (or [1][2d])."""
    theta, x = np.asarray(theta, np.float64), np.clip(np.asarray(x, np.float64), X_LO, X_HI)
    a, b = theta[:, 0::2], theta[:, 1::2]
    lx = np.log(x)
    om = -np.expm1(a * lx)
    l = np.sum(np.log(a) + np.log(b) + (a - 1.0) * lx + (b - 1.0) * np.log(om), axis=1)
    g = np.empty((x.shape[0], 2 * x.shape[1]))
    g[:, 0::2] = 1.0 / a + lx * (1.0 - (b - 1.0) * np.exp(a * lx) / om)
    g[:, 1::2] = 1.0 / b + np.log(om)
    terms = np.empty_like(g)
    terms[:, 0::2] = 1.0 / a + np.abs(lx) + np.abs((b - 1.0) * lx * np.exp(a * lx) / om)
    terms[:, 1::2] = 1.0 / b + np.abs(np.log(om))
    return l, g, terms


def group_advantage(reward, mask=None, normalise=True, eps=1e-6):
    r = np.asarray(reward, np.float64)
    m = np.ones(r.shape, bool) if mask is None else np.asarray(mask) != 0
    out = np.zeros(r.shape)
    for i in range(r.shape[0]):
        v = r[i, m[i]]
        if v.size:
            dev = v - v.mean()
            out[i, m[i]] = dev / (np.sqrt(np.mean(dev * dev)) + eps) if normalise else dev
    return out


def policy_loss(theta, theta_old, x, adv, theta_ref=None, mask=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                average="events"):
    """dict(loss, kl, clip_frac, dtheta, abs_dtheta): the last is the sum of the terms' absolute
    values, for condition-aware comparison, with an event's slope dL/dl taken as a whole (it may
    itself be a small rest of the ratio's and the divergence's)."""
    theta = np.asarray(theta, np.float64)
    R, E, d = x.shape
    m = np.ones((R, E), bool) if mask is None else np.asarray(mask) != 0
    n = m.sum(1)
    out = dict(loss=0.0, kl=0.0, clip_frac=0.0, dtheta=np.zeros((R, 2 * d)), abs_dtheta=np.zeros((R, 2 * d)))
    total = n.sum() if average == "events" else (n > 0).sum()
    for i in range(R):
        if not n[i]:
            continue
        w = 1.0 / total if average == "events" else 1.0 / (total * n[i])
        xi, A = x[i][m[i]], np.asarray(adv, np.float64)[i][m[i]]
        l, g, terms = event_logp(theta[i:i + 1], xi)
        rho = np.exp(l - event_logp(np.asarray(theta_old, np.float64)[i:i + 1], xi)[0])
        held = np.clip(rho, 1.0 - clip_low, 1.0 + clip_high)
        cut = held * A < rho * A
        val, slope = -np.minimum(rho * A, held * A), np.where(cut, 0.0, -rho * A)
        if theta_ref is not None:
            r = event_logp(np.asarray(theta_ref, np.float64)[i:i + 1], xi)[0] - l
            k = np.expm1(r) - r
            val, slope = val + kl_coef * k, slope - kl_coef * np.expm1(r)
            out["kl"] += w * k.sum()
        out["loss"] += w * val.sum()
        out["clip_frac"] += w * cut.sum()
        out["dtheta"][i] = w * slope @ g
        out["abs_dtheta"][i] = w * np.abs(slope) @ terms
    return out


def _softplus(t):
    return np.maximum(t, 0.0) + np.log1p(np.exp(-np.abs(t)))


def preference_loss(theta, theta_ref, chosen, rejected, len_chosen=None, len_rejected=None, beta=0.1,
                    label_smoothing=0.0):
    """dict(loss, margin, dtheta, abs_dtheta)."""
    theta, theta_ref = np.asarray(theta, np.float64), np.asarray(theta_ref, np.float64)
    R, P, d = theta.shape[0], chosen.shape[0], theta.shape[1] // 2
    margin, dtheta, ab = np.zeros(P), np.zeros((R, 2 * d)), np.zeros((R, 2 * d))
    for p in range(P):
        i = p // (P // R)
        S, Sabs, h = np.zeros(2 * d), np.zeros(2 * d), 0.0
        for sets, lens, sign in ((chosen, len_chosen, 1.0), (rejected, len_rejected, -1.0)):
            k = sets.shape[1] if lens is None else min(max(int(lens[p]), 0), sets.shape[1])
            l, g, terms = event_logp(theta[i:i + 1], sets[p, :k])
            h += sign * np.sum(l - event_logp(theta_ref[i:i + 1], sets[p, :k])[0])
            S += sign * g.sum(0)
            Sabs += terms.sum(0)
        margin[p] = beta * h
        slope = (label_smoothing - np.exp(-_softplus(margin[p]))) * beta / P     # sigmoid(h) - 1 + s
        dtheta[i] += slope * S
        ab[i] += abs(slope) * Sabs
    loss = np.mean((1.0 - label_smoothing) * _softplus(-margin) + label_smoothing * _softplus(margin))
    return dict(loss=loss, margin=margin, dtheta=dtheta, abs_dtheta=ab)


NS_COEF = (3.4445, -4.7750, 2.0315)


def orthogonalise(u, steps=5, coef=NS_COEF, eps=1e-7):
    """Newton-Schulz steps on the matrices u [...][rows][cols], shorter side as rows (Jordan et al.
    2024): stated on the singular values, which the odd polynomial a s + b s^3 + c s^5 acts on."""
    U, s, Vt = np.linalg.svd(np.asarray(u, np.float64), full_matrices=False)
    s = s / (np.sqrt(np.sum(s * s, axis=-1, keepdims=True)) + eps)
    a, b, c = coef
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return (U * s[..., None, :]) @ Vt


def muon_step(p, g, m, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale="shape", steps=5, coef=NS_COEF, eps=1e-7):
    """(p, m) after one step on matrices of any stack shape."""
    p, g = np.asarray(p, np.float64), np.asarray(g, np.float64)
    m = momentum * np.asarray(m, np.float64) + g
    o = orthogonalise(g + momentum * m if nesterov else m, steps, coef, eps)
    rows, cols = p.shape[-2:]
    s = {"none": 1.0, "shape": max(1.0, rows / cols) ** 0.5, "rms": 0.2 * max(rows, cols) ** 0.5}[scale]
    return (1.0 - lr * weight_decay) * p - lr * s * o, m
