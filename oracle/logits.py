"""What lies between a head's logits and the gradient that enters the network again, in float64 numpy from the definitions:
log probabilities of given tokens with entropy and the largest logits, distillation from a teacher's top logits, the
gradients of both.  Shares no code with the library."""
import numpy as np


def rows(z, tau=1.0):
    """(ln p [rows, cols], lse, entropy, bad, none): bad rows hold a NaN or +infinity, rows of none -infinity alone."""
    y = np.asarray(z, np.float64) / tau
    bad = (np.isnan(y) | (y == np.inf)).any(1)
    none = ~bad & (y == -np.inf).all(1)
    lp, lse, entropy = np.full(y.shape, np.nan), np.full(len(y), np.nan), np.full(len(y), np.nan)
    lp[none], lse[none], entropy[none] = -np.inf, -np.inf, 0.0
    for r in np.flatnonzero(~bad & ~none):
        top = y[r].max()
        log_sum = np.log(np.exp(y[r] - top).sum())
        lse[r] = top + log_sum
        lp[r] = (y[r] - top) - log_sum                    # (logits near the range's ends: the sum is lost in lse)
        p = np.exp(lp[r])
        entropy[r] = -(p[p > 0] * lp[r][p > 0]).sum()
    return lp, lse, entropy, bad, none


def logprobs(z, tokens, tau=1.0):
    """(logprob, entropy, lse)"""
    lp, lse, entropy, _, _ = rows(z, tau)
    out = np.zeros(len(lp))
    for r, t in enumerate(tokens):
        if t >= 0:
            out[r] = lp[r, t] if t < lp.shape[1] else np.nan
    return out, entropy, lse


def largest(z, k):
    """Ids of the k largest of each row, equal ones by their id."""
    return np.argsort(-np.asarray(z, np.float64), axis=1, kind="stable")[:, :k]


def logprobs_gradient(z, tokens, g, h=None, tau=1.0, lse=None, entropy=None):
    """lse, entropy: as a forward pass left them; the exact ones without."""
    lp, own_lse, own_entropy, bad, none = rows(z, tau)
    if lse is not None:
        with np.errstate(invalid="ignore"):
            lp = np.asarray(z, np.float64) / tau - np.asarray(lse, np.float64)[:, None]
        lp[bad] = np.nan
    entropy = own_entropy if entropy is None else entropy
    d = np.zeros(lp.shape)
    for r, t in enumerate(tokens):
        if none[r] or (t < 0 and h is None):
            continue
        p = np.exp(lp[r])
        if t >= 0:
            if t >= lp.shape[1]:
                d[r] = np.nan
                continue
            d[r] = -g[r] * p
            d[r, t] += g[r]
        if h is not None:
            d[r] -= h[r] * np.where(p > 0, p * (np.where(p > 0, lp[r], 0.0) + entropy[r]), p)
    return d / tau


def teacher(ids, values, tau=1.0, lse=None, cols=None):
    """q [rows, kept], 0 where there is no id; all NaN in rows with an id out of range, a value that is no number, or shares whose sum
    is beyond 32 bits' range."""
    ids, y = np.asarray(ids), np.asarray(values, np.float64) / tau
    q = np.zeros(y.shape)
    for r in range(len(y)):
        live = ids[r] >= 0
        if (ids[r] >= cols).any() or np.isnan(y[r][live]).any() or (y[r][live] == np.inf).any():
            q[r] = np.nan
        elif lse is not None:
            with np.errstate(invalid="ignore", over="ignore"):
                q[r][live] = np.exp(y[r][live] - lse[r])
            if not q[r].sum() <= np.finfo(np.float32).max:
                q[r] = np.nan
        elif live.any() and y[r][live].max() > -np.inf:
            e = np.exp(y[r][live] - y[r][live].max())
            q[r][live] = e / e.sum()
    return q


def distill(z, ids, values, tau=1.0, teacher_lse=None):
    """(loss, lse)"""
    lp, lse, _, bad, _ = rows(z, tau)
    q = teacher(ids, values, tau, teacher_lse, lp.shape[1])
    loss = np.zeros(len(lp))
    for r in range(len(lp)):
        for j in range(q.shape[1]):
            if np.isnan(q[r, j]):
                loss[r] = np.nan
            elif q[r, j] > 0:
                loss[r] += q[r, j] * (np.log(q[r, j]) - lp[r, ids[r, j]])
    return loss, lse


def distill_gradient(z, ids, values, g=None, tau=1.0, teacher_lse=None, lse=None):
    lp, _, _, bad, none = rows(z, tau)
    if lse is not None:
        with np.errstate(invalid="ignore"):
            lp = np.asarray(z, np.float64) / tau - np.asarray(lse, np.float64)[:, None]
        lp[bad] = np.nan
    q = teacher(ids, values, tau, teacher_lse, lp.shape[1])
    d = np.zeros(lp.shape)
    for r in range(len(lp)):
        if none[r] or not (q[r] != 0).any():
            continue
        d[r] = q[r].sum() * np.exp(lp[r])
        for j in np.flatnonzero(q[r] > 0):
            d[r, ids[r, j]] -= q[r, j]
        d[r] *= 1.0 if g is None else g[r]
    return d / tau
