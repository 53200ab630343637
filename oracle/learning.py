"""Definitions, in 64 bits and row by row, of what is learned from drawn tokens: log probabilities, the clipped policy loss and the loss over
pairs of answers, each with the slope of the loss with the log probability and the gradient of the logits."""
import math

import numpy as np


def row(logits, target):
    """(log probability of the target, max, sum of exp(l - max), probabilities, mean distance from the largest) of one row of finite or -infinite logits;
    None for a target outside the vocabulary."""
    V = len(logits)
    if not 0 <= target < V:
        return None
    l = logits.astype(np.float64)
    top = l.max()
    w = np.exp(l - top)
    total = math.fsum(w)
    d = np.where(w > 0, top - np.where(np.isfinite(l), l, top), 0.0)
    return l[target] - top - math.log(total), top, total, w / total, float((d * w).sum() / total)


def gradient(p, target, logp, slope):
    """slope * (one-hot - p), the target's entry without cancellation."""
    d = -slope * p
    d[target] = -slope * math.expm1(logp)
    return d


def policy_token(logp, old, adv, low, high, kl=0.0, ref=0.0):
    """(loss, slope) of one token."""
    r = math.exp(logp - old)
    bounded = min(max(r, 1.0 - low), 1.0 + high)
    loss, slope = (-r * adv, -r * adv) if r * adv <= bounded * adv else (-bounded * adv, 0.0)
    if kl:
        d = ref - logp
        loss += kl * (math.expm1(d) - d)
        slope -= kl * math.expm1(d)
    return loss, slope


def pair(chosen, rejected, beta, smooth, pairs):
    """(loss of a pair whose answers are `chosen` and `rejected` above their references, slope of the mean over `pairs` with chosen)."""
    delta = beta * (chosen - rejected)
    loss = sum(f * np.logaddexp(0.0, x) for f, x in ((1.0 - smooth, -delta), (smooth, delta)) if f)  # a factor of 0 leaves nothing of an infinite term
    sigma = 1.0 / (1.0 + math.exp(-delta)) if delta >= 0 else math.exp(delta) / (1.0 + math.exp(delta))
    return float(loss), -beta / pairs * ((1.0 - smooth) * (1.0 - sigma) - smooth * sigma)
