"""Drawing tokens, the first K of a row, and distillation from such lists.  TEST INFRASTRUCTURE ONLY.

Plain fp64 restatements, row by row, of the formulas in include/pods.h (pods_sample, pods_topk, pods_distill_chunk); the
sampling policy is the one whose log-probabilities L_GRPO and L_PODS take as old_logp (Sections 3.1, 3.2).  Pinned in
tests/test_oracle_rollout.py.
"""
import numpy as np

GREEDY_BELOW = 2.0 ** -20


def order(row):
    """Ids by larger logit, then lower id."""
    return np.lexsort((np.arange(row.shape[0]), -(row + 0.0)))


def sample_row(row, u, tau=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row of logits (float64).  Returns dict(token, logp, logq, kept (ids in order), edge): edge is the distance of
    the drawn point u * S from the nearest boundary between two tokens and of top_p's goal from the nearest prefix sum, as a
    share of S - a draw with a tiny edge is not decided by the formula but by rounding."""
    row = np.asarray(row, np.float64)
    if np.isnan(row).any() or (row == np.inf).any():
        return dict(token=-1, logp=np.nan, logq=np.nan, kept=np.zeros(0, np.int64), edge=np.inf)
    if (row == -np.inf).all():
        return dict(token=-1, logp=-np.inf, logq=-np.inf, kept=np.zeros(0, np.int64), edge=np.inf)
    greedy = tau < GREEDY_BELOW
    if greedy:
        tau = 1.0
    d = (row - row.max()) / tau
    e = np.exp(d)
    ids = order(row)
    if greedy:
        return dict(token=int(ids[0]), logp=d[ids[0]] - np.log(e.sum()), logq=0.0, kept=ids[:1], edge=np.inf)
    V = row.shape[0]
    count = V if top_k <= 0 or top_k >= V else int(top_k)
    edge = np.inf
    if top_p < 1.0:
        run = np.cumsum(e[ids[:count]])
        goal = top_p * run[-1]
        if goal > 0:
            edge = min(edge, float(np.abs(run - goal).min() / run[-1]))
        reach = np.nonzero(run >= goal)[0]
        p_count = int(reach[0]) + 1 if len(reach) else count
    else:
        p_count = count
    # e >= min_p, asked of the exponents: exp rounds to 1 what lies just below
    m_count = int((d >= np.log(min(min_p, 1.0))).sum()) if min_p > 0 else V
    kept = ids[:max(1, min(count, p_count, m_count))]
    by_id = np.sort(kept)
    run = np.cumsum(e[by_id])
    target = u * run[-1]
    # at u = 0 every finite logit counts, also where fp64 has no weight left for it
    at = int(np.nonzero(row[by_id] > -np.inf)[0][0]) if u == 0 else int(np.nonzero(run > target)[0][0])
    inner = run[:-1]
    if target > 0 and len(inner):
        edge = min(edge, float(np.abs(inner - target).min() / run[-1]))
    token = int(by_id[at])
    return dict(token=token, logp=d[token] - np.log(e.sum()), logq=d[token] - np.log(run[-1]), kept=kept, edge=edge)


def topk_row(row, K, tau=1.0):
    """dict(ids [K], values [K], lse)."""
    row = np.asarray(row, np.float64)
    if np.isnan(row).any() or (row == np.inf).any():
        return dict(ids=np.full(K, -1), values=np.full(K, np.nan), lse=np.nan)
    ids = order(row)[:K]
    m = row.max()
    lse = -np.inf if m == -np.inf else m / tau + np.log(np.exp((row - m) / tau).sum())
    return dict(ids=ids, values=row[ids], lse=lse)


def distill_row(row, ids, values, teacher_lse=None, tau=1.0, rest=False):
    """kl of one row and its gradient with respect to the logits (weights and grad_scale left out), and terms [V]: the sum
    of the absolute values of the gradient's terms, the scale its rounding errors are relative to."""
    row = np.asarray(row, np.float64)
    V = row.shape[0]
    ids = np.asarray(ids, np.int64)
    use = (ids >= 0) & (ids < V)
    ids, y = ids[use], np.asarray(values, np.float64)[use] / tau
    if np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
        return dict(kl=np.nan, grad=np.full(V, np.nan), terms=np.full(V, np.nan), Q=np.nan, r=0.0)
    if teacher_lse is None:
        L = 0.0
        if len(y) and y.max() > -np.inf:
            L = y.max() + np.log(np.exp(y - y.max()).sum())
    else:
        L = float(teacher_lse)
    lq = y - L
    q = np.exp(lq)
    Q = q.sum()
    d = (row - row.max()) / tau
    e = np.exp(d)
    logp = d - np.log(e.sum())
    p = np.exp(logp)
    outside = np.ones(V, bool)
    outside[ids] = False
    away = p[outside].sum()
    r = max(0.0, 1.0 - Q) if rest and (row[outside] > -np.inf).any() else 0.0
    live = q > 0
    kl = float((q[live] * (lq[live] - logp[ids[live]])).sum())
    grad = (Q + r) * p
    terms = (Q + r) * p
    if r > 0:
        m2 = d[outside].max()                              # 1 - s without underflow
        e2 = np.exp(d[outside] - m2)
        log_away = m2 + np.log(e2.sum()) - np.log(e.sum())
        kl += r * (np.log(r) - log_away)
        grad[outside] -= r * e2 / e2.sum()
        terms[outside] += r * e2 / e2.sum()
    np.subtract.at(grad, ids, q)
    np.add.at(terms, ids, q)
    return dict(kl=kl, grad=grad, terms=terms, Q=Q, r=r, away=away)
