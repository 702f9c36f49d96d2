"""fp64 oracle of token log-probabilities from logits with their gradient, and of the pair losses on packed rollouts.

Written from the formulas in include/pods.h, a row and a pair at a time.  (The paper has no counterpart.)"""
import math

import numpy as np


def log_softmax(z, temperature):
    """float64 row; relative to the largest logit, so that a common offset of any size takes nothing away."""
    z = np.asarray(z, np.float64)
    d = (z - z.max()) / float(temperature)
    return d - math.log(np.exp(d).sum())


def logp_row(z, token, temperature):
    """z: float64 row -> (logp, lse, entropy)."""
    z = np.asarray(z, np.float64)
    top = z.max()
    if np.isnan(z).any() or top == np.inf:
        return math.nan, math.nan, math.nan
    if top == -np.inf:
        return math.nan, -math.inf, math.nan
    logq = log_softmax(z, temperature)
    live = logq > -700
    return float(logq[token]), float(top / temperature - logq.max()), float(-(np.exp(logq[live]) * logq[live]).sum())


def logp_grad_row(z, token, temperature, dlogp, dentropy=0.0):
    """d (dlogp logp + dentropy entropy) / dz."""
    logq = log_softmax(z, temperature)
    entropy = logp_row(z, token, temperature)[2]
    p = np.exp(logq)
    g = -dlogp * p
    live = p > 0
    g[live] -= dentropy * p[live] * (logq[live] + entropy)
    g[token] += dlogp
    return g / float(temperature)


def pair_loss(h, kind, smoothing, beta):
    """(loss, d loss / dh)."""
    if kind == "sigmoid":
        def nls(x):                                    # -log sigma(x)
            return max(-x, 0.0) + math.log1p(math.exp(-abs(x)))

        def sig(x):
            return 1.0 / (1.0 + math.exp(-x)) if x >= 0 else math.exp(x) / (1.0 + math.exp(x))
        loss, slope = (1.0 - smoothing) * nls(h), -(1.0 - smoothing) * sig(-h)
        if smoothing:
            loss, slope = loss + smoothing * nls(-h), slope + smoothing * sig(h)
        return loss, slope
    if kind == "hinge":
        return max(0.0, 1.0 - h), -1.0 if h < 1.0 else 0.0
    return ((h - 0.5) / beta) ** 2, 2.0 * (h - 0.5) / beta ** 2


def preference(logp, ref_logp, mask, cu, pairs, beta, kind="sigmoid", smoothing=0.0, margin=0.0, pair_weight=None,
               average=False, nll=0.0, grad_scale=1.0):
    """(loss, dlogp [T], reward [M], pair_loss [P]) in fp64; margin a number or [P]."""
    logp = np.asarray(logp, np.float64)
    T, M, P = logp.shape[0], len(cu) - 1, len(pairs)
    mask = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    ref = np.zeros(T) if ref_logp is None else np.asarray(ref_logp, np.float64)
    margin = np.broadcast_to(np.asarray(margin, np.float64), (P,))
    rows = [[t for t in range(cu[i], cu[i + 1]) if mask[t]] for i in range(M)]
    score = np.array([math.fsum(logp[t] - ref[t] for t in r) / (len(r) if average and r else 1) for r in rows])
    like = np.array([-math.fsum(logp[t] for t in r) / len(r) if r else 0.0 for r in rows])
    ok = [0 <= c < M and 0 <= r < M for c, r in pairs]
    w = np.full(P, 1.0 / max(1, sum(ok))) if pair_weight is None else np.asarray(pair_weight, np.float64)
    losses, dscore, dlike = np.zeros(P), np.zeros(M), np.zeros(M)
    for p, (c, r) in enumerate(pairs):
        if not ok[p]:
            continue
        losses[p], slope = pair_loss(beta * (score[c] - score[r]) - margin[p], kind, smoothing, beta)
        losses[p] += nll * like[c]
        dscore[c] += w[p] * slope * beta
        dscore[r] -= w[p] * slope * beta
        dlike[c] += w[p] * nll
    dlogp = np.zeros(T)
    for i, r in enumerate(rows):
        for t in r:
            dlogp[t] = grad_scale * (dscore[i] / (len(r) if average else 1) - dlike[i] / len(r))
    return float((w * losses * ok).sum()), dlogp, beta * score, losses
