"""Plain fp64 numpy forms of the operators at a model's dense ends, for the
tests: embedding and gradient, log probabilities behind a dense head and
gradients, norm and clipping.  Written from their definitions; shares no code
with the kernels."""
from __future__ import annotations

import numpy as np


def embedding(table, ids, scale):
    """Rows of the table; an id outside it gives zeros."""
    table, ids = np.asarray(table, np.float64), np.asarray(ids)
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < len(table):
            out[t] = scale * table[i]
    return out


def embedding_backward(grad, ids, vocab, scale):
    """(gradient of the table, sum of the absolute values of its terms, tokens of each row)."""
    grad, ids = np.asarray(grad, np.float64), np.asarray(ids)
    out, size, count = np.zeros((vocab, grad.shape[1])), np.zeros((vocab, grad.shape[1])), np.zeros(vocab, np.int64)
    for t, i in enumerate(ids):
        if 0 <= i < vocab:
            out[i] += scale * grad[t]
            size[i] += abs(scale) * np.abs(grad[t])
            count[i] += 1
    return out, size, count


def linear(x, weight, scale):
    """(logits, sums of the absolute values of their terms)."""
    x, weight = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    return scale * (x @ weight.T), scale * (np.abs(x) @ np.abs(weight).T)


def softmax_moments(z):
    """lse, entropy and probabilities of each row."""
    top = z.max(-1, keepdims=True)
    top = np.where(np.isneginf(top), 0.0, top)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.exp(z - top)
        total = e.sum(-1, keepdims=True)
        lse = np.log(total) + top
        p = np.where(np.isneginf(lse), 0.0, e / total)
        entropy = lse[:, 0] - np.where(p > 0, p * np.where(p > 0, z, 0.0), np.where(np.isnan(p), np.nan, 0.0)).sum(-1)
    return lse[:, 0], np.where(np.isneginf(lse[:, 0]), 0.0, entropy), p


def logits_gradient(z, targets, g_logprob, g_entropy):
    """Gradient for the logits: rows without a target have no g_logprob, rows without gradients none at all."""
    rows, vocab = z.shape
    lse, entropy, p = softmax_moments(z)
    out = np.zeros_like(z)
    for r in range(rows):
        asked = targets is not None and 0 <= targets[r] < vocab
        g = float(g_logprob[r]) if asked and g_logprob is not None else 0.0
        ge = float(g_entropy[r]) if g_entropy is not None else 0.0
        if g == 0 and ge == 0:
            continue
        lp = np.where(p[r] > 0, z[r] - lse[r], 0.0)
        out[r] = -g * p[r] - ge * p[r] * (lp + entropy[r])
        if g != 0:
            out[r, targets[r]] += g
    return out


def clip(tensors, max_norm):
    """(norm, clipped tensors)."""
    tensors = [np.asarray(t, np.float64) for t in tensors]
    norm = float(np.sqrt(sum(float((t * t).sum()) for t in tensors)))
    factor = 1.0 if norm == 0 else min(1.0, max_norm / norm)
    return norm, [t * factor for t in tensors]
