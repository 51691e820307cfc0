"""Plain numpy definitions, in 64 bits, of the row operators: the embedding
lookup and its gradient, log probabilities with entropy and alternatives, and
the distillation loss with its gradient (CPU, test infrastructure only; shares
no code with the HIP path)."""
from __future__ import annotations

import numpy as np


def embed_lookup(table, ids, scale):
    """out[i] = scale * sum_j table[ids[i, j]]; ids outside the table count 0."""
    table = np.asarray(table, dtype=np.float64)
    out = np.zeros((ids.shape[0], table.shape[1]))
    for i in range(ids.shape[0]):
        for j in ids[i]:
            if 0 <= j < table.shape[0]:
                out[i] += table[j]
    return scale * out


def embed_gradient(grad, ids, rows, scale):
    grad = np.asarray(grad, dtype=np.float64)
    out = np.zeros((rows, grad.shape[1]))
    for i in range(ids.shape[0]):
        for j in ids[i]:
            if 0 <= j < rows:
                out[j] += grad[i]
    return scale * out


def row_length(n_valid, i, cols):
    return cols if n_valid is None else int(np.clip(n_valid[i], 0, cols))


def log_softmax(x, tau):
    """log softmax(x / tau) of one row; None where it has no distribution, NaN
    throughout where a logit is NaN or +inf."""
    x = np.asarray(x, dtype=np.float64)
    if np.isnan(x).any() or np.isposinf(x).any():
        return np.full(x.shape, np.nan)
    if x.size == 0 or np.isneginf(x).all():
        return None
    z = (x - x.max()) / tau
    return z - np.log(np.exp(z).sum())


def log_probs(logits, tau=1.0, n_valid=None, given=None, n_top=0):
    """(given_out, entropy, top_ids, top) as ifvs_log_probs defines them."""
    n, cols = logits.shape
    n_given = 0 if given is None else given.shape[1]
    given_out = np.full((n, n_given), -np.inf)
    entropy = np.zeros(n)
    top_ids = np.full((n, n_top), -1, dtype=np.int64)
    top = np.full((n, n_top), -np.inf)
    for i in range(n):
        m = row_length(n_valid, i, cols)
        x = np.asarray(logits[i, :m], dtype=np.float64)
        lp = log_softmax(x, tau)
        if lp is not None and np.isnan(lp).any():
            entropy[i] = np.nan
            top[i] = np.nan
        elif lp is not None:
            p = np.exp(lp)
            entropy[i] = -(p[p > 0] * lp[p > 0]).sum()
            order = np.lexsort((np.arange(m), -x))
            order = order[~np.isneginf(x[order])][:n_top]
            top_ids[i, :order.size] = order
            top[i, :order.size] = lp[order]
        for g in range(n_given):
            if 0 <= given[i, g] < m:
                given_out[i, g] = -np.inf if lp is None else lp[given[i, g]]
    return given_out, entropy, top_ids, top


def distill(logits, teacher_ids, teacher_logits, tau=1.0, teacher_lse=None, row_weight=None, n_valid=None):
    """(loss [n], row_weight * dloss / dlogits [n, cols])."""
    n, cols = logits.shape
    loss = np.zeros(n)
    grad = np.zeros((n, cols))
    for i in range(n):
        w = 1.0 if row_weight is None else float(row_weight[i])
        if w == 0.0:
            continue
        m = row_length(n_valid, i, cols)
        lq = log_softmax(logits[i, :m], tau)
        there = [k for k in range(teacher_ids.shape[1]) if 0 <= teacher_ids[i, k] < m]
        t = np.asarray(teacher_logits[i, there], dtype=np.float64)
        at = np.asarray(teacher_ids[i, there], dtype=np.int64)
        if lq is None or (teacher_lse is None and not there):
            # left out whatever the teacher's sum is; a NaN or +inf still shows
            bad_teacher = np.isnan(t).any() or np.isposinf(t).any()
            if not bad_teacher:
                continue
            lq = np.full(m, np.nan)
        if teacher_lse is None:
            lp = log_softmax(t, tau)
            lp = np.full(t.shape, np.nan) if lp is None else lp
        else:
            lp = t / tau - float(teacher_lse[i])
            if np.isposinf(t).any() or not np.isfinite(teacher_lse[i]):
                lp = np.full(t.shape, np.nan)
        if np.isnan(lp).any() or np.isnan(lq).any() or (teacher_lse is not None and not np.isfinite(teacher_lse[i])):
            loss[i] = np.nan
            grad[i, :m] = np.nan
            continue
        p = np.exp(lp)
        q = np.exp(lq)
        with np.errstate(divide="ignore", invalid="ignore"):
            value = np.where(p > 0, p * (lp - lq[at]), 0.0).sum()
            target = np.zeros(m)
            np.add.at(target, at, p)
            if teacher_lse is not None:
                named = np.zeros(m, dtype=bool)
                named[at] = True
                left = max(0.0, 1.0 - p.sum())
                lq_rest = lq[~named]
                lq_rest = lq_rest[~np.isneginf(lq_rest)]
                if lq_rest.size:             # else no other column to give the rest to
                    # shares from differences: far below the row's maximum a
                    # logarithm no longer holds that of their sum
                    e = np.exp(lq[~named] - lq_rest.max())
                    if left > 0:
                        value += left * (np.log(left) - (lq_rest.max() + np.log(e.sum())))
                    target[~named] = left * (e / e.sum())
        loss[i] = tau * tau * value
        grad[i, :m] = w * tau * (q - target)
    return loss, grad
