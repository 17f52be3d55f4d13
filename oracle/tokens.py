"""Answers over a vocabulary in 64 bits, row by row from the definitions in
``include/rafiki_tokens.h``: the combined distribution, sampling, top-k, distillation with its
gradient, and the 8-bit FC layer.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

P_MIN = 2.0 ** -1000
REST_MIN = 2.0 ** -20


def combined(z, t):
    """Mean over models of softmax(z / t) for one row, z [S, C]; classes below 2^-1000 are 0.  None: a model's
    row is empty (all -inf); NaN: NaN or +inf in it, or no temperature."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or (z == np.inf).any() or not t >= 0:
        return math.nan
    top = z.max(1, keepdims=True)
    if (top == -np.inf).any():
        return None
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.where(z == -np.inf, -np.inf, (z - top) / (t if t > 0 else 1.0))
        e = np.exp(x)
    p = (e / e.sum(1, keepdims=True)).mean(0)
    p[p < P_MIN] = 0
    return p


def ranked(p):
    """Classes with a probability, by p down and index up."""
    order = np.argsort(-p, kind="stable")
    return order[p[order] > 0]


def sample(z, u, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(label, probability) of one row z [S, C]."""
    p = combined(z, t)
    if p is None:
        return -1, 0.0
    if isinstance(p, float):
        return -1, math.nan
    order = ranked(p)
    if t == 0:
        return int(order[0]), 1.0
    if top_k > 0:
        order = order[:top_k]
    if top_p < 1:
        reached = np.cumsum(p[order])
        order = order[:1 + int((reached < float(top_p) * reached[-1]).sum())] if top_p > 0 else order[:1]
    if min_p > 0:
        order = order[p[order] >= min(float(min_p), 1.0) * p[order[0]]]
    kept = np.sort(order)
    reached = np.cumsum(p[kept])
    if u >= 1:
        j = kept.size - 1
    else:
        j = int((reached <= (float(u) if u > 0 else 0.0) * reached[-1]).sum())
    return int(kept[j]), p[kept[j]] / reached[-1]


def topk(z, k, t=1.0):
    """(labels [k], logp [k]) of one row z [S, C]."""
    labels, logp = np.full(k, -1, np.int32), np.full(k, -np.inf)
    p = combined(z, t)
    if isinstance(p, float):
        logp[:] = math.nan
    elif p is not None:
        order = ranked(p)[:k]
        labels[:order.size], logp[:order.size] = order, np.log(p[order])
    return labels, logp


def _lse(x):
    top = x.max() if x.size else -np.inf
    return top + math.log(np.exp(x - top).sum()) if top > -np.inf else -np.inf


def distill(z, labels, logp, t=1.0, rest=False, g=1.0):
    """(loss, gradient [C]) of one row z [C] against the slots (labels, logp)."""
    z = np.asarray(z, np.float64)
    C = z.size
    q = np.zeros(C)
    member = np.zeros(C, bool)
    valid = (labels >= 0) & (labels < C)
    logp = np.asarray(logp, np.float64)
    if not rest and valid.any():
        total = _lse(logp[valid]) if not np.isnan(logp[valid]).any() else math.nan
        if total == -np.inf:
            valid = np.zeros_like(valid)
        else:
            logp = logp - total
    if not rest and not valid.any():
        return 0.0, np.zeros(C)
    np.add.at(q, labels[valid], np.exp(logp[valid]))
    member[labels[valid]] = True
    x = z / t
    if np.isnan(x).any() or np.isnan(q).any() or x.max() in (np.inf, -np.inf):
        return math.nan, np.zeros(C) if g == 0 else np.full(C, math.nan)
    lse = _lse(x)
    with np.errstate(divide="ignore"):
        lx, lq = x - lse, np.log(q)
    loss = (q[q > 0] * (lq[q > 0] - lx[q > 0])).sum()
    q_r, share = 0.0, np.zeros(C)
    if rest:
        q_r = 1 - q.sum()
        if q_r < REST_MIN or member.all():
            q_r = 0.0
        lr = _lse(x[~member]) if (~member).any() else -np.inf
        if q_r > 0:
            loss += q_r * (math.log(q_r) - (lr - lse)) if lr > -np.inf else math.inf
        if lr > -np.inf:
            share[~member] = np.exp(x[~member] - lr)
        else:
            q_r = 0.0                   # p_r = 0: no class can take it, and the gradient is that of the others
    d = (q.sum() + q_r) * np.exp(lx) - q - q_r * share
    return t * t * loss, t * g * d if g != 0 else np.zeros(C)


def quantize_rows(x):
    """(q, scale fp32) of rows x [n, c] fp32: an fp32 quotient's neighbours in 64 bits decide every tie."""
    top = np.abs(x.astype(np.float64)).max(1)
    bad = ~np.isfinite(x).all(1)
    scale = (np.where(bad, 1, top).astype(np.float32) / np.float32(127)).astype(np.float32)
    scale[scale < np.float32(2.0 ** -126)] = 0
    s = np.where(scale == 0, 1, scale).astype(np.float64)[:, None]
    q = np.rint(np.where(bad[:, None], 0, x).astype(np.float64) / s) * (scale > 0)[:, None]
    return q.astype(np.int8), np.where(bad, np.float32(np.nan), scale)


def fc_i8(x, sx, w, sw, bias=None, relu=False):
    y = (x.astype(np.float64) @ w.astype(np.float64).T) * (sx.astype(np.float64)[:, None] * sw.astype(np.float64))
    y = y + (0 if bias is None else bias.astype(np.float64))
    return np.maximum(y, 0) if relu else y
