"""The operators on rows of logits, written out in 64 bits with numpy: what the GPU tests compare with."""
import numpy as np


def order(x):
    """Allowed actions of one row: falling logit, lower index first among equal ones."""
    ids = np.nonzero(x > -np.inf)[0]
    return ids[np.argsort(-x[ids], kind="stable")]


def weights(x, ids, temperature):
    top = x[ids[0]]
    if np.isinf(top):
        return (x[ids] == top).astype(np.float64)
    with np.errstate(over="ignore"):
        return np.exp(-((top - x[ids]) / temperature))


def choose(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(kept actions in order, their inclusive sums, place of the choice in them); None: nothing is allowed."""
    x = np.asarray(x, np.float64)
    ids = order(x)
    if not len(ids):
        return None
    if not temperature > 0:
        return ids[:1], np.ones(1), 0
    if 0 < top_k < len(ids):
        ids = ids[:top_k]
    w = weights(x, ids, temperature)
    c = np.cumsum(w)
    before = np.concatenate([[0.0], c[:-1]])
    keep = np.ones(len(ids), bool)
    if top_p < 1:
        keep &= before < top_p * c[-1]
    if min_p > 0:
        keep &= w >= min_p
    keep[0] = True
    count = int(np.argmin(keep)) if not keep.all() else len(keep)
    c = c[:count]
    at = int(np.searchsorted(c, (u if u > 0 else 0.0) * c[-1], side="right"))
    return ids[:count], c, min(at, count - 1)


def log_sum_exp(x, temperature=1.0):
    z = np.asarray(x, np.float64) / temperature
    z = z[z > -np.inf]
    return -np.inf if not len(z) else z.max() + np.log(np.exp(z - z.max()).sum())


def distill(x, t, index, weight=1.0, teacher_lse=None, ts=1.0, tt=1.0):
    """Loss and gradient of one row, entry by entry, and how far 32-bit exponentials may move each of them.

    The kernel's exponentials are exp2 of a 32-bit product of a 32-bit difference: each is off by at most
    2^-23 of its exponent and 2^-23 of itself, a sum over a row by the weighted mean of that, where the mean
    exponent is at most log(n) + 1; log, quotients and the entries' terms are in 64 bits."""
    x, t = np.asarray(x, np.float64), np.asarray(t, np.float64)
    n = len(x)
    g, slack = np.zeros(n), np.zeros(n)
    if weight == 0:
        return 0.0, g, 0.0, slack
    there = (index >= 0) & (index < n)
    t, j = t[there] / tt, np.asarray(index)[there]
    lse = log_sum_exp(x, ts)
    if lse == -np.inf or (teacher_lse is None and not (t > -np.inf).any()):
        return 0.0, g, 0.0, slack
    z = x / ts
    p = np.exp(z - lse)
    log_q = t - (log_sum_exp(t) if teacher_lse is None else teacher_lse)
    q = np.exp(log_q)
    live = q > 0
    loss = (q[live] * (log_q[live] - (z[j][live] - lse))).sum()
    named = np.zeros(n, bool)
    named[j] = True
    total = q.sum()
    unit = 2.0 ** -22 * (np.log(n) + 4)
    loss_slack = unit * total
    reach = np.full(n, total)
    if teacher_lse is not None:
        p_rest, q_rest = p[~named].sum(), 1 - total
        if q_rest > 0 and p_rest > 0:
            loss += q_rest * (np.log(q_rest) - np.log(p_rest))
            loss_slack += unit * q_rest
            total = 1.0
            reach = np.where(named, 1.0, 1.0 + (q.sum() + p[named].sum()) / p_rest)
            g[~named] -= q_rest / p_rest * p[~named]
    g += p * total
    np.subtract.at(g, j, q)
    taken = np.zeros(n)
    np.add.at(taken, j, q)
    depth = np.where(p > 0, lse - np.where(p > 0, z, 0.0), 0.0)
    slack = p * reach * (unit + 2.0 ** -22 * np.abs(depth)) + 2.0 ** -24 * taken
    scale = abs(weight) / ts
    return loss * weight, g * (weight / ts), loss_slack * abs(weight) + 2.0 ** -23 * abs(loss * weight), slack * scale


def distill_rest(x, t, index, teacher_lse, ts, tt, weight=1.0):
    """distill with a teacher's log-sum-exp, from logarithms alone, for students whose mass outside the entries is
    as small as it may be: (loss, gradient, slack of the loss, slack of the gradient) of one row.

    The kernel's weight of an action without an entry is made from a maximum that is at most 46 + log n student temperatures
    above the largest of them (a sum of 1e-20 or more is kept).  It is off by three roundings of its distance to that maximum,
    under 2^-22 of it, and by under 2^-22 of itself; their sum by the mean of that, of at most log n more, and with it p_rest, the
    total and every logarithm of them.  Weights below 2^-126 are 0: 2^-126 / 1e-20 of the sum at most."""
    x, t, n = np.asarray(x, np.float64), np.asarray(t, np.float64), len(x)
    there = (index >= 0) & (index < n)
    t, j = t[there] / tt, np.asarray(index)[there]
    named = np.zeros(n, bool)
    named[j] = True
    # (from the maximum: a log-sum-exp of 1e30 would lose the log of a sum)
    out = named | (x == -np.inf)
    top, own = x.max(), x[~out].max() if not out.all() else -np.inf
    z = (x - top) / ts
    depth = np.zeros(n) if out.all() else np.where(out, 0.0, own - np.where(out, own, x)) / ts
    total, rest = np.exp(z).sum(), np.exp(-depth)[~out].sum()
    log_rest = -np.inf if out.all() else (own - top) / ts + np.log(rest) - np.log(total)
    share = np.where(out, 0.0, np.exp(-depth) / max(rest, 1e-300))
    log_q = t - teacher_lse
    q = np.exp(log_q)
    a, live = q.sum(), q > 0
    q_rest, p_rest = 1 - a, np.exp(log_rest)
    p = np.exp(z) / total
    loss = (q[live] * (log_q[live] - (z[j][live] - np.log(total)))).sum()
    reached = q_rest > 0 and log_rest > -np.inf
    if reached:
        loss += q_rest * (np.log(q_rest) - log_rest)
    inside, pull = (1.0, p_rest - q_rest) if reached else (a, a * p_rest)
    taken = np.zeros(n)
    np.add.at(taken, j, q)
    g = np.where(named, p * inside - taken, share * pull)
    unit = 2.0 ** -22 * (2 * 46 + 3 * np.log(n) + 8)
    slack = np.where(named, (p * inside + taken) * unit, share * ((unit + 2.0 ** -22 * depth) * (abs(pull) + p_rest) + 2.0 ** -48)
                     + 2.0 ** -126 / 1e-20 * abs(pull))
    loss_slack = unit * (a + abs(q_rest)) + 2.0 ** -23 * abs(loss) + 2.0 ** -46 * (q[live] * np.abs(x[j][live] / ts)).sum()
    scale = abs(weight) / ts
    return loss * weight, g * (weight / ts), loss_slack * abs(weight), slack * scale
