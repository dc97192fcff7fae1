"""The operators on a router's logits from their formulas, row by row quantities in numpy's 64-bit floats.

Shares nothing with the GPU path.  Every function takes the logits as float64 (exact images of the fp32, bf16 or fp16
values) and returns float64; `counts` says which rows count: not masked, and with a logit above -infinity.
"""
from __future__ import annotations

import numpy as np


def rows_that_count(x, row_mask=None):
    some = ~np.all(x == -np.inf, axis=1)
    return some if row_mask is None else some & (np.asarray(row_mask) != 0)


def softmax(x, tau=1.0, row_mask=None):
    """(z, p, lse) of the rows that count; zeros elsewhere."""
    live = rows_that_count(x, row_mask)
    z = np.where(live[:, None], x, 0.0) / tau
    with np.errstate(invalid="ignore"):
        top = np.max(z, axis=1, keepdims=True)
        e = np.exp(z - top)
    total = e.sum(axis=1, keepdims=True)
    lse = (top + np.log(total))[:, 0]
    return live, z, np.where(live[:, None], e / total, 0.0), np.where(live, lse, 0.0)


def _safe_log(p):
    return np.log(np.where(p > 0, p, 1.0))


def logprobs(x, topk_idx, m=0, tau=1.0, row_mask=None):
    live, z, p, lse = softmax(x, tau, row_mask)
    E = x.shape[1]
    good = live[:, None] & (topk_idx >= 0) & (topk_idx < E)
    at = np.clip(topk_idx, 0, E - 1)
    logp = np.where(good, np.take_along_axis(z, at, 1) - lse[:, None], 0.0)
    with np.errstate(invalid="ignore"):
        log_p = np.where((z > -np.inf) | np.isnan(z), z - lse[:, None], 0.0)
        entropy = np.where(live, -(p * log_p).sum(axis=1), 0.0)
    order = np.argsort(-x, axis=1, kind="stable")[:, :m]
    value = np.take_along_axis(x, order, 1)
    there = live[:, None] & (value > -np.inf)
    alt_idx = np.where(there, order, -1)
    alt_logp = np.where(there, value / tau - lse[:, None], np.where(live[:, None], -np.inf, 0.0))
    return logp, lse, entropy, alt_idx, alt_logp


def logprobs_backward(x, topk_idx, d_logp, d_lse, d_entropy, tau=1.0, row_mask=None):
    """(gradient, the magnitudes its terms add up to)"""
    live, z, p, lse = softmax(x, tau, row_mask)
    E = x.shape[1]
    good = live[:, None] & (topk_idx >= 0) & (topk_idx < E)
    g = np.where(good, d_logp, 0.0)
    log_p = np.where(z > -np.inf, z - lse[:, None], 0.0)
    h = -(p * log_p).sum(axis=1)
    spread = np.zeros_like(x)
    many = np.zeros_like(x)
    rows = np.arange(x.shape[0])
    for j in range(topk_idx.shape[1]):
        at = np.clip(topk_idx[:, j], 0, E - 1)
        spread[rows, at] += g[:, j]
        many[rows, at] += np.abs(g[:, j])
    pull = g.sum(axis=1) - d_lse
    dx = spread - p * (pull[:, None] + d_entropy[:, None] * (log_p + h[:, None]))
    size = many + p * (np.abs(g).sum(axis=1) + np.abs(d_lse) + np.abs(d_entropy) * (np.abs(h) + 1.0))[:, None] + p * np.abs(d_entropy[:, None] * log_p)
    return np.where(live[:, None], dx, 0.0) / tau, np.where(live[:, None], size, 0.0) / tau


def balance(x, topk_idx, edges, coef, row_mask=None):
    """edges: list of (first row, end) of the groups."""
    live, _, p, _ = softmax(x, 1.0, row_mask)
    E, k = x.shape[1], topk_idx.shape[1]
    n = len(edges)
    counts, tokens = np.zeros((n, E), np.int64), np.zeros(n, np.int64)
    sums, loss = np.zeros((n, E)), np.zeros(n)
    for g, (a, b) in enumerate(edges):
        use = live[a:b]
        picks = topk_idx[a:b][use]
        picks = picks[(picks >= 0) & (picks < E)]
        counts[g] = np.bincount(picks, minlength=E)
        tokens[g] = use.sum()
        sums[g] = p[a:b].sum(axis=0)
        if tokens[g]:
            loss[g] = coef * E / (k * float(tokens[g]) ** 2) * (counts[g] * sums[g]).sum()
    return counts, tokens, sums, loss


def balance_backward(x, k, edges, coef, counts, tokens, d_loss, row_mask=None):
    """(gradient, magnitudes); NaN in the rows of no group"""
    live, _, p, _ = softmax(x, 1.0, row_mask)
    E = x.shape[1]
    dx, size = np.full_like(x, np.nan), np.zeros_like(x)
    for g, (a, b) in enumerate(edges):
        w = d_loss[g] * coef * E / (k * max(float(tokens[g]), 1.0) ** 2) * counts[g].astype(np.float64) * (tokens[g] > 0)
        w = w - w.mean()
        dot = (p[a:b] * w).sum(axis=1, keepdims=True)
        dx[a:b] = p[a:b] * (w - dot)
        size[a:b] = p[a:b] * (np.abs(w) + (p[a:b] * np.abs(w)).sum(axis=1, keepdims=True))
    return dx, size


def distill_terms(x, t_idx, t_logit, t_lse, tau=1.0, row_mask=None):
    live, z, p, lse = softmax(x, tau, row_mask)
    T, E = x.shape
    good = live[:, None] & (t_idx >= 0) & (t_idx < E) & (t_logit != -np.inf)
    at = np.where(good, t_idx, 0)
    u = np.where(good, t_logit / tau, -np.inf)
    if t_lse is None:
        top = np.where(good.any(axis=1), u.max(axis=1), 0.0)[:, None]
        log_mass = top[:, 0] + np.log(np.maximum(np.exp(u - top).sum(axis=1), 1e-300))
    else:
        log_mass = t_lse
    q = np.where(good, np.exp(u - log_mass[:, None]), 0.0)
    inside = np.zeros((T, E), bool)
    for j in range(t_idx.shape[1]):
        inside[np.arange(T)[good[:, j]], at[good[:, j], j]] = True
    rest_p = np.where(inside, 0.0, p).sum(axis=1)
    mass = q.sum(axis=1)
    rest_q = np.where((rest_p > 0) & live, np.maximum(1.0 - mass, 0.0), 0.0) if t_lse is not None else np.zeros(T)
    return dict(live=live & good.any(axis=1), z=z, p=p, lse=lse, good=good, at=at, u=u, log_mass=log_mass, q=q, inside=inside,
                rest_p=rest_p, rest_q=rest_q, mass=mass)


def distill(x, t_idx, t_logit, t_lse=None, tau=1.0, row_mask=None):
    o = distill_terms(x, t_idx, t_logit, t_lse, tau, row_mask)
    log_p = np.take_along_axis(o["z"], o["at"], 1) - o["lse"][:, None]
    log_q = np.where(o["good"], o["u"] - o["log_mass"][:, None], 0.0)
    terms = np.where(o["q"] > 0, o["q"] * (log_q - np.where(o["q"] > 0, log_p, 0.0)), 0.0).sum(axis=1)
    rest = np.where(o["rest_q"] > 0, o["rest_q"] * (_safe_log(o["rest_q"]) - _safe_log(o["rest_p"])), 0.0)
    return np.where(o["live"], tau * tau * (terms + rest), 0.0)


def distill_backward(x, t_idx, t_logit, d_loss, t_lse=None, tau=1.0, row_mask=None):
    """(gradient, magnitudes)"""
    o = distill_terms(x, t_idx, t_logit, t_lse, tau, row_mask)
    listed = np.zeros_like(x)
    for j in range(t_idx.shape[1]):
        listed[np.arange(x.shape[0]), o["at"][:, j]] += o["q"][:, j]
    whole = (o["mass"] + o["rest_q"])[:, None]
    ratio = np.where(o["rest_q"] > 0, o["rest_q"] / np.where(o["rest_p"] > 0, o["rest_p"], 1.0), 0.0)[:, None]
    dz = o["p"] * (whole - np.where(o["inside"], 0.0, ratio)) - listed
    size = o["p"] * (whole + np.where(o["inside"], 0.0, ratio)) + listed
    unit = np.where(o["live"], tau * d_loss, 0.0)[:, None]
    return dz * unit, size * np.abs(unit)
