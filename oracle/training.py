"""Plain float64 forms of the losses over rows of logits, the gradient norm and the update: written from
their definitions, one row, pair or tensor at a time, sharing no code with the package."""
from __future__ import annotations

import numpy as np


def row_distribution(z):
    """(log-probabilities, probabilities) of one row, or None if no class is possible (all logits -inf)."""
    z = np.asarray(z, np.float64)
    if np.all(z == -np.inf):
        return None
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.max(z)
        e = np.exp(z - top)
        s = np.sum(e)
        return z - top - np.log(s), e / s


def policy_loss(logits, actions, old_logp, advantages, *, ref_logp=None, weight=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0):
    """dict of loss, logp, kl, slope (d loss / d log p) per row and the gradient."""
    n, C = logits.shape
    out = {k: np.zeros(n) for k in ("loss", "logp", "kl", "slope")}
    out["grad"] = np.zeros((n, C))
    for r in range(n):
        w = 1.0 / n if weight is None else float(weight[r])
        a = int(actions[r])
        if w == 0.0 or not 0 <= a < C:
            continue
        dist = row_distribution(logits[r])
        if dist is None:
            continue
        lp, p = dist[0][a], dist[1]
        adv = float(advantages[r])
        ratio = np.exp(lp - float(old_logp[r]))
        free, held = -adv * ratio, -adv * min(max(ratio, 1 - clip_low), 1 + clip_high)
        if np.isnan(free):
            loss = slope = free
        else:
            loss, slope = max(free, held), free if free >= held else 0.0
        if ref_logp is not None:
            d = float(ref_logp[r]) - lp
            out["kl"][r] = np.inf if d == np.inf else np.expm1(d) - d
            if kl_coef:
                loss += kl_coef * out["kl"][r]
                slope -= kl_coef * np.expm1(d)
        out["loss"][r], out["logp"][r], out["slope"][r] = w * loss, lp, w * slope
        one = np.zeros(C)
        one[a] = 1.0
        out["grad"][r] = w * slope * (one - p) if slope else 0.0
    return out


def preference_loss(logits, actions, seq_ptr, *, ref_logp=None, weight=None, beta=0.1, smoothing=0.0):
    """dict of loss and margin per pair, logp and slope per row and the gradient."""
    n, C = logits.shape
    pairs = len(seq_ptr) // 2
    out = {"loss": np.zeros(pairs), "margin": np.zeros(pairs), "logp": np.zeros(n), "slope": np.zeros(n),
           "grad": np.zeros((n, C))}
    dists = {}
    for r in range(int(seq_ptr[0]), int(seq_ptr[-1])):
        a = int(actions[r])
        dist = row_distribution(logits[r]) if 0 <= a < C else None
        if dist is not None:
            dists[r] = dist[1]
            out["logp"][r] = dist[0][a]
    for p in range(pairs):
        w = 1.0 / pairs if weight is None else float(weight[p])
        rows = [range(int(seq_ptr[2 * p + k]), int(seq_ptr[2 * p + k + 1])) for k in (0, 1)]
        total = [sum(out["logp"][r] for r in rows[k]) - (0.0 if ref_logp is None else float(ref_logp[2 * p + k]))
                 for k in (0, 1)]
        h = beta * (total[0] - total[1])
        out["margin"][p] = h
        if w == 0.0:
            continue
        minus_log_sig = lambda x: np.logaddexp(0.0, -x)
        out["loss"][p] = w * sum(k * minus_log_sig(x) for k, x in ((1 - smoothing, h), (smoothing, -h)) if k)
        sig = lambda x: np.exp(-np.logaddexp(0.0, -x))
        slope = beta * w * (-(1 - smoothing) * sig(-h) + smoothing * sig(h))
        for k, sign in ((0, 1.0), (1, -1.0)):
            for r in rows[k]:
                if r in dists:
                    one = np.zeros(C)
                    one[int(actions[r])] = 1.0
                    out["slope"][r] = sign * slope
                    out["grad"][r] = sign * slope * (one - dists[r])
    return out


def grad_norm(grads):
    return float(np.sqrt(sum(float(np.sum(np.square(np.asarray(g, np.float64)))) for g in grads)))


def clip_factor(norm, max_norm):
    return max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0


def adamw(p, g, m, v, *, lr, beta1, beta2, eps, weight_decay, step, factor=1.0):
    """(p, m, v) after the step."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    g = factor * g
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    with np.errstate(invalid="ignore", divide="ignore"):
        change = (m / (1 - beta1 ** step)) / (np.sqrt(v / (1 - beta2 ** step)) + eps)
    return (1 - lr * weight_decay) * p - lr * change, m, v
