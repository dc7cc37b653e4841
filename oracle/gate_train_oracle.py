"""CPU oracle of the operators that train a gate: the balance loss and the expert counts it rests on, the routing
weights' gradient, the loss of a gate against the gate it predicts, the gate product's gradients, and the global
gradient norm with clipping.

TEST INFRASTRUCTURE ONLY, written from the formulas in NumPy fp64; it shares no code with the HIP sources.  The paper
fine-tunes copies of gates as load predictors (Section 4.1) and prints no formula for their loss: taken is the mean
Kullback-Leibler divergence from the target gate's softmax.  Pins: tests/test_gate_train_pins.py.
"""
from __future__ import annotations

import numpy as np


def softmax(scores):
    """Rows of probabilities in fp64; -inf is an expert that is switched off, and a row of nothing else is all zeros.  A NaN
    makes its row NaN."""
    s = np.asarray(scores, dtype=np.float64)
    m = s.max(axis=1, keepdims=True)
    e = np.exp(s - np.where(np.isneginf(m), 0.0, m))
    total = e.sum(axis=1, keepdims=True)
    return e / np.where(total == 0.0, 1.0, total)


def _real(token_mask, T):
    return np.arange(T) if token_mask is None else np.flatnonzero(token_mask)


def balance_loss(scores, topk_idx, token_mask=None):
    """(counts [E] int64, prob_sum [E], loss)."""
    T, E = scores.shape
    rows = _real(token_mask, T)
    k = topk_idx.shape[1]
    counts = np.zeros(E, dtype=np.int64)
    for e in topk_idx[rows].ravel():
        if 0 <= e < E:
            counts[e] += 1
    prob_sum = softmax(scores[rows]).sum(axis=0) if rows.size else np.zeros(E)
    total = counts.sum()
    loss = 0.0 if total == 0 else E * k * float((counts * prob_sum).sum()) / float(total) ** 2
    return counts, prob_sum, loss


def routing_weights(scores, topk_idx, renorm):
    """softmax over all experts read at the chosen ones, renormalised or not; 0 for indices that name no expert."""
    p = softmax(scores)
    E = scores.shape[1]
    ok = (topk_idx >= 0) & (topk_idx < E)
    w = np.where(ok, np.take_along_axis(p, np.where(ok, topk_idx, 0).astype(np.int64), axis=1), 0.0)
    if renorm:
        s = np.where(ok, np.take_along_axis(np.asarray(scores, dtype=np.float64), np.where(ok, topk_idx, 0).astype(np.int64), axis=1), -np.inf)
        w = softmax(s)
    return w


def route_backward(scores, topk_idx, d_topk_w, counts, balance_coef, renorm, token_mask=None, k=None):
    """Gradient of sum d_topk_w * topk_w + balance_coef * loss(counts fixed); rows of padded tokens are 0."""
    T, E = scores.shape
    out = np.zeros((T, E))
    rows = _real(token_mask, T)
    if rows.size == 0:
        return out
    p = softmax(scores[rows])
    g = np.zeros_like(p)
    d = np.zeros_like(p)
    if counts is not None:
        total = float(np.sum(counts, dtype=np.int64))
        kk = topk_idx.shape[1] if k is None else k
        if total > 0:
            g += balance_coef * E * kk * np.asarray(counts, dtype=np.float64)[None, :] / total ** 2
    if d_topk_w is not None:
        dw = np.asarray(d_topk_w, dtype=np.float64)[rows]
        idx = topk_idx[rows]
        w = routing_weights(scores[rows], idx, renorm)
        inner = (w * dw * ((idx >= 0) & (idx < E))).sum(axis=1) if renorm else None
        for i in range(rows.size):
            for j in range(idx.shape[1]):
                e = idx[i, j]
                if not 0 <= e < E:
                    continue
                if renorm:
                    d[i, e] += w[i, j] * (dw[i, j] - inner[i])
                else:
                    g[i, e] += dw[i, j]
    out[rows] = d + p * (g - (p * g).sum(axis=1, keepdims=True))
    return out


def gate_distill(scores, target_scores, coef=1.0, token_mask=None):
    """(mean KL(q || p) over the tokens that count, coef / N (p - q))."""
    T, E = scores.shape
    rows = _real(token_mask, T)
    grad = np.zeros((T, E))
    if rows.size == 0:
        return 0.0, grad
    p, q = softmax(scores[rows]), softmax(target_scores[rows])
    left = (p.sum(axis=1) != 0) & (q.sum(axis=1) != 0)
    loss = 0.0
    for i in np.flatnonzero(left):
        s, t = np.asarray(scores[rows[i]], dtype=np.float64), np.asarray(target_scores[rows[i]], dtype=np.float64)
        log_p = s - s.max() - np.log(np.exp(s - s.max()).sum())
        log_q = t - t.max() - np.log(np.exp(t - t.max()).sum())
        on = q[i] != 0
        loss += float((q[i][on] * (log_q[on] - log_p[on])).sum())
    grad[rows[left]] = coef / rows.size * (p[left] - q[left])
    return loss / rows.size, grad


def gate_backward(x, w_gate, d_scores, token_mask=None):
    """(d_w_gate [E,d], d_gate_bias [E], d_x [T,d]) of score = x w_gate^T + bias; x and w_gate in fp64."""
    rows = _real(token_mask, x.shape[0])
    ds = np.asarray(d_scores, dtype=np.float64)[rows]
    d_x = np.zeros(x.shape)
    d_x[rows] = ds @ w_gate
    return ds.T @ x[rows], ds.sum(axis=0), d_x


def clip_grads(grads, max_norm):
    """(norm over all tensors, the tensors times min(1, max_norm / norm)); unscaled if the norm is not finite."""
    with np.errstate(over="ignore", invalid="ignore"):
        norm = float(np.sqrt(sum(float(np.square(np.asarray(g, dtype=np.float64)).sum()) for g in grads)))
    c = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, [np.asarray(g, dtype=np.float64) * c for g in grads]
