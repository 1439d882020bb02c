"""Oracle of what stands between tokens and an 8-bit output layer, and between its gradient and the optimiser: norms with the
residual's addition and their adjoint, embeddings and their gradient, clipping by the norm of all gradients, adjusted logits.

TEST INFRASTRUCTURE ONLY: plain numpy in 64 bits from the definitions; the product path (the HIP library) shares no code
with it.  Where a bound on rounding errors needs it, the sum over magnitudes is returned beside the sum.
"""
import numpy as np


def rms_norm(x, residual, weight, eps):
    """(h, y)"""
    h = np.asarray(x, np.float64) if residual is None else np.asarray(x, np.float64) + residual
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h, h * r * (1.0 if weight is None else np.asarray(weight, np.float64))


def rms_norm_backward(dy, h, weight, eps, d_h=None):
    """(dx, d_weight, magnitude of dx's terms, magnitude of d_weight's terms)"""
    dy, h = np.asarray(dy, np.float64), np.asarray(h, np.float64)
    g = dy * (1.0 if weight is None else np.asarray(weight, np.float64))
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    u = h * r
    dx = r * (g - u * (g * u).mean(1, keepdims=True))
    mag = r * (np.abs(g) + np.abs(u) * np.abs(g * u).mean(1, keepdims=True))
    if d_h is not None:
        dx, mag = dx + d_h, mag + np.abs(d_h)
    return dx, (dy * u).sum(0), mag, np.abs(dy * u).sum(0)


def embedding(table, ids, scale):
    table, ids = np.asarray(table, np.float64), np.asarray(ids)
    ok = (ids >= 0) & (ids < len(table))
    return np.where(ok[:, None], table[np.where(ok, ids, 0)] * scale, 0.0)


def embedding_backward(d_out, ids, vocab, scale):
    """(gradient, the same sum over magnitudes, how many terms)"""
    d_out, ids = np.asarray(d_out, np.float64), np.asarray(ids)
    ok = (ids >= 0) & (ids < vocab)
    grad, mag, n = np.zeros((vocab, d_out.shape[1])), np.zeros((vocab, d_out.shape[1])), np.bincount(ids[ok], minlength=vocab)
    for i in np.flatnonzero(ok):
        grad[ids[i]] += d_out[i]
        mag[ids[i]] += np.abs(d_out[i])
    return grad * scale, mag * abs(scale), n


def grad_clip(grads, max_norm):
    """(norm, clipped gradients)"""
    grads = [np.asarray(g, np.float64) for g in grads]
    norm = np.sqrt(sum((g * g).sum() for g in grads))
    factor = max_norm / norm if norm > max_norm and np.isfinite(norm) else 1.0
    return norm, [g * factor for g in grads]


def logits_adjust(z, history=None, n_prompt=None, repetition=None, presence=None, frequency=None, bias_id=None, bias=None, allowed=None):
    """(adjusted logits, magnitude of the terms); one token at a time, in the order of the definition"""
    out = np.array(z, np.float64)
    rows, vocab = out.shape
    mag = np.abs(out)
    for r in range(rows):
        if history is not None:
            tokens = [(i, int(t)) for i, t in enumerate(history[r]) if 0 <= t < vocab]
            first = 0 if n_prompt is None else int(n_prompt[r])
            count = {}
            for i, t in tokens:
                if i >= first:
                    count[t] = count.get(t, 0) + 1
            rep = 1.0 if repetition is None else float(repetition[r])
            for t in {t for _, t in tokens}:
                out[r, t] = out[r, t] / rep if out[r, t] > 0 else out[r, t] * rep
                mag[r, t] = abs(out[r, t])
            for t, c in count.items():
                off = (0.0 if frequency is None else float(frequency[r])) * c
                more = 0.0 if presence is None else float(presence[r])
                out[r, t] = out[r, t] - off - more
                mag[r, t] += abs(off) + abs(more)
        if bias_id is not None:
            for t, b in {int(t): float(b) for t, b in zip(bias_id[r], bias[r])}.items():      # the last entry of a token stays
                if 0 <= t < vocab:
                    out[r, t] += b
                    mag[r, t] += abs(b)
        if allowed is not None:
            j = np.arange(vocab)
            out[r, (np.asarray(allowed[r]).astype(np.int64)[j // 32] >> (j % 32)) & 1 == 0] = -np.inf
    return out, mag
