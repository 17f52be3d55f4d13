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


# ---------------------------------------------------------------- losses over given tokens

def token_facts(z, y, t=1.0):
    """(log p_y, H, p, log p) of one row z [C] of logits, or None where it has no distribution."""
    x = np.asarray(z, np.float64) / t
    if np.isnan(x).any() or x.max() in (np.inf, -np.inf):
        return None
    top = x.max()
    e = np.exp(x - top)
    rest = np.delete(e, np.argmax(x)).sum()              # the sum without its 1: log1p keeps what is small
    log_p = (x - top) - math.log1p(rest)
    p = np.exp(log_p)
    return log_p[y], -(p[p > 0] * log_p[p > 0]).sum(), p, log_p


def token_grad(z, y, t, a, h=0.0):
    """Gradient of a log p_y + h H by the row z."""
    facts = token_facts(z, y, t)
    if a == 0 and h == 0:
        return np.zeros(len(z))
    if facts is None or not math.isfinite(a) or math.isnan(h):
        return np.full(len(z), math.nan)
    _, H, p, log_p = facts
    others = np.delete(p, y).sum()
    d = -a * p
    d[y] = a * others
    if h:
        d -= h * np.where(p > 0, p * (np.where(p > 0, log_p, 0.0) + H), 0.0)
    return d / t


def policy(z, y, A, old=None, ref=None, t=1.0, low=0.2, high=0.2, kl_coef=0.0, ent_coef=0.0, g=1.0):
    """(loss, log p, kl, H, gradient) of one row."""
    C = len(z)
    if not 0 <= y < C:
        return 0.0, 0.0, 0.0, 0.0, np.zeros(C)
    facts = token_facts(z, y, t)
    if facts is None:
        return (math.nan,) * 4 + (np.zeros(C) if g == 0 else np.full(C, math.nan),)
    logp, H = facts[:2]
    fp32 = lambda v: math.inf if v > 3.5e38 else v  # noqa: E731
    loss = kl = slope = 0.0
    with np.errstate(all="ignore"):
        if A != 0:
            r = fp32(np.exp(np.float64(logp) - old)) if old is not None else 1.0
            plain = r * np.float64(A)
            cut = np.clip(r, 1 - low, 1 + high) * np.float64(A)
            loss = math.nan if np.isnan(plain) else -min(plain, cut)
            slope = math.nan if np.isnan(plain) else (-plain if plain <= cut else 0.0)
        if ref is not None:
            d = np.float64(ref) - logp
            e = fp32(np.exp(d))
            kl = math.inf if e == math.inf else np.expm1(d) - d
            if kl_coef:
                loss += kl_coef * kl
                slope -= kl_coef * (math.inf if e == math.inf else np.expm1(d))
    if ent_coef:
        loss -= ent_coef * H
    if g == 0:
        return loss, logp, kl, H, np.zeros(C)
    bad = math.isnan(loss) or not math.isfinite(slope)
    return loss, logp, kl, H, np.full(C, math.nan) if bad else token_grad(z, y, t, g * slope, -g * ent_coef)


def preference(z, labels, offsets, ref=None, t=1.0, beta=0.1, smoothing=0.0, mean=False, g=None):
    """(loss [P], scores [P, 2], gradient [n, C]; rows of no answer are NaN there) of rows z [n, C]."""
    n, C = z.shape
    P = (len(offsets) - 1) // 2
    losses, scores, grad = np.zeros(P), np.zeros((P, 2)), np.full((n, C), math.nan)
    soft = lambda v: max(v, 0.0) + math.log1p(math.exp(-abs(v)))  # noqa: E731
    sig = lambda v: 1 / (1 + math.exp(-v)) if v > -700 else 0.0  # noqa: E731
    for p in range(P):
        count = [0, 0]
        for k in range(2):
            total = 0.0
            for i in range(offsets[2 * p + k], offsets[2 * p + k + 1]):
                if 0 <= labels[i] < C:
                    facts = token_facts(z[i], labels[i], t)
                    total += (math.nan if facts is None else facts[0]) - (0.0 if ref is None else float(ref[i]))
                    count[k] += 1
            scores[p, k] = beta * (total / count[k] if mean and count[k] else total)
        u = scores[p, 0] - scores[p, 1]
        if math.isnan(u):
            losses[p] = du = math.nan
        else:
            losses[p] = (1 - smoothing) * soft(-u) + (smoothing * soft(u) if smoothing else 0.0)
            du = smoothing * sig(u) - (1 - smoothing) * sig(-u)
        gp = 1.0 if g is None else float(g[p])
        for k in range(2):
            a = 0.0 if gp == 0 else (-1 if k else 1) * beta * gp * du / (count[k] if mean and count[k] else 1)
            for i in range(offsets[2 * p + k], offsets[2 * p + k + 1]):
                grad[i] = token_grad(z[i], labels[i], t, a) if 0 <= labels[i] < C else 0.0
    return losses, scores, grad


# ---------------------------------------------------------------- 4-bit floating point in blocks

MX4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6])


def quantize_mx4(x):
    """(codes [n, 32 b], bytes [n, b]) of rows x [n, c] fp32: the nearest magnitude, a tie to the even code."""
    n, c = x.shape
    v = np.zeros((n, (c + 31) // 32 * 32))
    v[:, :c] = x
    v = v.reshape(n, -1, 32)
    with np.errstate(invalid="ignore"):
        top = np.abs(v).max(2)
    bad = ~np.isfinite(v).all(2)
    exponent = np.frexp(np.where(bad | (top == 0), 2.0 ** -140, top))[1] - 1
    e = np.maximum(exponent - 2, -127)
    u = np.abs(np.where(bad[..., None], 0, v)) / np.exp2(e.astype(np.float64))[..., None]
    away = np.abs(u[..., None] - MX4[:8])
    nearest = away.min(-1, keepdims=True)
    order = [0, 2, 4, 6, 1, 3, 5, 7]                         # even codes are asked first
    code = np.array(order)[(away[..., order] == nearest).argmax(-1)]
    code = code + 8 * (np.signbit(v) & ~bad[..., None])
    return code.reshape(n, -1).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def mx4_values(codes, scale):
    """What codes [n, 32 b] and bytes [n, b] stand for."""
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return (MX4[codes].reshape(codes.shape[0], -1, 32) * s[..., None]).reshape(codes.shape)


def fc_mx4(x, xs, w, ws, bias=None, relu=False):
    y = mx4_values(x, xs) @ mx4_values(w, ws).T + (0 if bias is None else bias.astype(np.float64))
    return np.maximum(y, 0) if relu else y
