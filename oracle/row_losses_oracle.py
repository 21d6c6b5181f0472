"""The losses on rows of logits in 64 bits, written from their definitions
(include/pgc.h, "losses on rows of logits"): loops over rows and sequences,
numpy only.  Each function also gives the gradient from its formula; the
formulas are checked against differences of the losses in the tests.
"""

from __future__ import annotations

import numpy as np


def rows(x, y, tau=1.0):
    """(logp, m, L, p) of every row: p softmax(x / tau); zeros in a row without a target, NaN
    for a target that is no class or a row without a distribution."""
    x = np.asarray(x, np.float64)
    T, V = x.shape
    logp, m, L, p = np.zeros(T), np.zeros(T), np.zeros(T), np.zeros((T, V))
    with np.errstate(all="ignore"):
        for t in range(T):
            if y[t] < 0:
                continue
            m[t] = x[t].max()
            e = np.exp((x[t] - m[t]) / tau)
            L[t] = np.log(e.sum())
            p[t] = e / e.sum()
            logp[t] = (x[t, y[t]] - m[t]) / tau - L[t] if y[t] < V else np.nan
    return logp, m, L, p


def logits_gradient(x, y, coef, tau=1.0):
    """coef_t (one_hot(y_t) - p_t) / tau; zeros where there is no target or coef is 0."""
    _, _, _, p = rows(x, y, tau)
    g = np.zeros_like(p)
    for t in range(len(y)):
        if y[t] < 0 or coef[t] == 0:
            continue
        g[t] = -coef[t] * p[t] / tau
        if y[t] < p.shape[1]:
            g[t, y[t]] += coef[t] / tau
        else:
            g[t] = np.nan
    return g


def preference(x, y, off, ref=None, beta=0.1, kind="sigmoid", margin=0.0, smoothing=0.0, average=False, scale=1.0,
               tau=1.0):
    """(loss, scores [pairs][2], coef [rows])"""
    logp, _, _, _ = rows(x, y, tau)
    pairs = (len(off) - 1) // 2
    coef, scores, total = np.zeros(len(y)), np.zeros((pairs, 2)), 0.0
    for i in range(pairs):
        share = []
        for j in range(2):
            t = [t for t in range(off[2 * i + j], off[2 * i + j + 1]) if y[t] >= 0]
            share.append(1.0 / max(len(t), 1) if average else 1.0)
            scores[i, j] = sum(logp[q] for q in t) * share[j]
        r = np.zeros(2) if ref is None else np.asarray(ref[i], np.float64)
        h = beta * ((scores[i, 0] - r[0]) - (scores[i, 1] - r[1])) - margin
        e = smoothing
        if kind == "sigmoid":
            f = (1 - e) * np.logaddexp(0, -h) + e * np.logaddexp(0, h)
            df = e * np.exp(-np.logaddexp(0, -h)) - (1 - e) * np.exp(-np.logaddexp(0, h))     # e sig(h) - (1 - e) sig(-h)
        elif kind == "hinge":
            f = (1 - e) * max(0.0, 1 - h) + e * max(0.0, 1 + h)
            df = e * (h > -1) - (1 - e) * (h < 1)
        else:
            a, b = h / beta - 0.5 / beta, h / beta + 0.5 / beta
            f = (1 - e) * a * a + e * b * b
            df = 2 / beta * ((1 - e) * a + e * b)
        total += scale * f / pairs
        for j in range(2):
            for t in range(off[2 * i + j], off[2 * i + j + 1]):
                if y[t] >= 0:
                    coef[t] = (1, -1)[j] * scale * beta * df / pairs * share[j]
    return total, scores, coef


def policy_weights(y, reduction, off=None):
    w = np.zeros(len(y))
    if reduction == "sequences":
        held = [[t for t in range(a, b) if y[t] >= 0] for a, b in zip(off[:-1], off[1:])]
        full = sum(len(h) > 0 for h in held)
        for h in held:
            for t in h:
                w[t] = 1.0 / (len(h) * full)
    else:
        n = sum(v >= 0 for v in y)
        w[np.asarray(y) >= 0] = 1.0 if reduction == "sum" else 1.0 / max(n, 1)
    return w


def policy(x, y, old, adv, ref=None, clip=(0.2, 0.2), kl=0.0, off=None, reduction="tokens", scale=1.0, tau=1.0):
    """(loss, terms [3], logp, coef)"""
    logp, _, _, _ = rows(x, y, tau)
    w = policy_weights(y, reduction, off)
    coef, terms = np.zeros(len(y)), np.zeros(3)
    for t in range(len(y)):
        if w[t] == 0:
            continue
        r = np.exp(logp[t] - float(old[t]))
        A = float(adv[t])
        q = min(max(r, 1.0 - float(np.float32(clip[0]))), 1.0 + float(np.float32(clip[1])))
        clipped = q * A < r * A
        terms[0] += w[t] * (0.0 if A == 0 else -min(r * A, q * A))
        terms[2] += w[t] * clipped
        slope = 0.0 if clipped else -r * A
        if ref is not None:
            u = float(ref[t]) - logp[t]
            terms[1] += w[t] * (np.expm1(u) - u)
            slope -= kl * np.expm1(u)
        coef[t] = scale * w[t] * slope
    return scale * (terms[0] + kl * terms[1]), terms, logp, coef


def balance(x, k, mask=None, choice=None, alpha=0.01):
    """(loss, counts, choice, gradient)"""
    x = np.asarray(x, np.float64)
    T, E = x.shape
    on = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    if choice is None:
        choice = np.full((T, k), -1, np.int32)
        for t in np.flatnonzero(on):
            order = sorted((e for e in range(E) if x[t, e] > -np.inf), key=lambda e: (-x[t, e], e))[:k]
            choice[t, :len(order)] = order
    counts = np.zeros(E, np.int64)
    for t in np.flatnonzero(on):
        for e in choice[t]:
            if 0 <= e < E:
                counts[e] += 1
    n = max(int(on.sum()), 1)
    w = alpha * E / (k * n * n) * counts
    loss, g = 0.0, np.zeros_like(x)
    for t in np.flatnonzero(on):
        if x[t].max() == -np.inf:
            continue
        with np.errstate(all="ignore"):
            p = np.exp(x[t] - x[t].max())
            p /= p.sum()
        loss += w @ p
        g[t] = p * (w - w @ p)
    return loss, counts, choice, g
