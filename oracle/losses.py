"""TEST INFRASTRUCTURE.  Losses on stored logits beyond cross-entropy, in 64 bits and row by row from their definitions: distillation from a
teacher's words, the clipped policy loss with a divergence term, and the preference loss on pairs.  Gradients are the formulas'; the tests hold
them to differences of the losses.  A row of weight 0 is not looked at.
"""
from __future__ import annotations

import numpy as np


def log_sum_exp(z):
    m = z.max()
    if not np.isfinite(m):
        return np.nan if m > 0 or np.isnan(m) else -np.inf
    return m + np.log(np.exp(z - m).sum())


def softmax(z):
    return np.exp(z - log_sum_exp(z))


def distill_row(z, ids, teacher, target, tau, soft, hard):
    """(loss, gradient, log-sum-exp of z / tau, log-sum-exp of z); a term that is off or has no used slot is left out."""
    z = np.asarray(z, dtype=np.float64)
    loss, grad, lses = 0.0, np.zeros_like(z), [0.0, 0.0]
    if soft:
        lses[0] = log_sum_exp(z / tau)
        used = [(i, float(t)) for i, t in zip(ids, teacher) if 0 <= i < len(z)]
        if used and max(t for _, t in used) > -np.inf:
            q = softmax(np.array([t for _, t in used]) / tau)
            grad += soft * tau * np.exp(z / tau - lses[0])
            for (i, _), qk in zip(used, q):
                if qk > 0:
                    loss += soft * tau * tau * qk * (np.log(qk) - (z[i] / tau - lses[0]))
                grad[i] -= soft * tau * qk
    if hard:
        lses[1] = log_sum_exp(z)
        loss += hard * (lses[1] - z[target])
        grad += hard * softmax(z)
        grad[target] -= hard
    return loss, grad, lses[0], lses[1]


def policy_of_logp(logp, old, ref, advantage, clip_low, clip_high, kl_weight):
    """(loss, derivative by logp)"""
    ratio = np.exp(logp - old)
    plain, clipped = ratio * advantage, min(max(ratio, 1 - clip_low), 1 + clip_high) * advantage
    loss, d = -min(plain, clipped), -plain if plain <= clipped else 0.0
    if kl_weight:
        e = ref - logp
        loss += kl_weight * (np.expm1(e) - e)
        d -= kl_weight * np.expm1(e)
    return loss, d


def token_logp(z, target):
    """(logp, lse, gradient of logp by z)"""
    z = np.asarray(z, dtype=np.float64)
    lse = log_sum_exp(z)
    grad = -np.exp(z - lse)
    grad[target] += 1.0
    return z[target] - lse, lse, grad


def preference_of_margin(margin, kind, beta, smoothing):
    """(loss, derivative by the margin)"""
    h = beta * margin
    if kind == "sigmoid":
        return ((1 - smoothing) * np.logaddexp(0.0, -h) + smoothing * np.logaddexp(0.0, h), beta * (smoothing - 1.0 / (1.0 + np.exp(h))))
    if kind == "hinge":
        return max(0.0, 1.0 - h), -beta if h < 1.0 else 0.0
    off = margin - 0.5 / beta
    return off * off, 2.0 * off
