"""Oracle of the passes over logits: log probabilities with entropy and top alternatives, and the divergence from a
teacher's top logits with its gradient.

TEST INFRASTRUCTURE ONLY: plain numpy float64, row by row from the definitions
  q_j = exp(z_j / T) / sum_k exp(z_k / T);   H = -sum q log q;
  L = sum_i p_i log(p_i / q_{c_i}) + p_r log(p_r / q_r),   dL/dz_j = (P q_j - p_j) / T in the list, q_j (P - p_r / q_r) / T outside.
"""
import numpy as np


def log_softmax(z, temperature=1.0):
    """(log q, lse) of one row; a row without anything above -inf has -inf everywhere."""
    x = np.asarray(z, dtype=np.float64) / temperature
    if np.isnan(x).any() or np.isposinf(x).any():
        return np.full_like(x, np.nan), np.nan
    m = x.max()
    if m == -np.inf:
        return x.copy(), -np.inf
    log_sum = np.log(np.exp(x - m).sum())
    return (x - m) - log_sum, m + log_sum                  # not x - lse: next to a maximum of 1e38 nothing is left of log_sum


def token_logprobs(z, tokens=None, top_k=0, temperature=1.0):
    """dict(lse, entropy, logprob, top_id, top_logit, top_logprob) of rows of logits; tokens [rows][n]."""
    z = np.asarray(z, dtype=np.float64)
    rows, vocab = z.shape
    n = 0 if tokens is None else tokens.shape[1]
    out = dict(lse=np.empty(rows), entropy=np.empty(rows), logprob=np.zeros((rows, n)), top_id=np.empty((rows, top_k), np.int64),
               top_logit=np.empty((rows, top_k)), top_logprob=np.empty((rows, top_k)))
    for r in range(rows):
        logq, out["lse"][r] = log_softmax(z[r], temperature)
        some = logq > -np.inf
        out["entropy"][r] = np.nan if np.isnan(logq).any() else -(np.exp(logq[some]) * logq[some]).sum()
        for i in range(n):
            t = tokens[r, i]
            if 0 <= t < vocab:
                out["logprob"][r, i] = logq[t]
        order = np.lexsort((np.arange(vocab), -np.where(np.isnan(z[r]), 0, z[r]), np.isnan(z[r])))[:top_k]     # NaN last, then falling, then by index
        out["top_id"][r], out["top_logit"][r], out["top_logprob"][r] = order, z[r][order], logq[order]
    return out


def distill(z, top_id, top_logit, temperature=1.0, teacher_lse=None, weight=None):
    """(loss_rows, loss, gradient of loss)."""
    z = np.asarray(z, dtype=np.float64)
    rows, vocab = z.shape
    loss, grad = np.zeros(rows), np.zeros_like(z)
    w = np.ones(rows) if weight is None else np.asarray(weight, dtype=np.float64)
    for r in range(rows):
        if w[r] == 0:
            continue
        logq, lse = log_softmax(z[r], temperature)
        if lse == -np.inf:
            continue
        there = (top_id[r] >= 0) & (top_id[r] < vocab)
        ids, t = top_id[r][there], np.asarray(top_logit[r], dtype=np.float64)[there] / temperature
        if teacher_lse is not None:
            logp = t - float(teacher_lse[r])
        else:
            logp = log_softmax(t)[0] if len(t) else t
        p = np.exp(logp)
        outside = np.ones(vocab, bool)
        outside[ids] = False
        q = np.exp(logq)
        q_out = q[outside].sum()
        p_out = max(0.0, 1.0 - p.sum()) if teacher_lse is not None and q_out != 0 else 0.0
        mass = p.sum() + p_out
        with np.errstate(all="ignore"):
            loss[r] = sum(pi * (lp - lq) for pi, lp, lq in zip(p, logp, logq[ids]) if pi != 0)
            if p_out > 0:
                loss[r] += p_out * (np.log(p_out) - np.log(q_out))
            g = q * (mass - (p_out / q_out if p_out > 0 else 0.0))
        g[ids] = mass * q[ids] - p
        grad[r] = g * w[r] / temperature
    live = w != 0
    return loss, float((loss[live] * w[live]).sum()), grad
