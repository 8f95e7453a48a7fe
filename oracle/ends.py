"""The operators at the two ends of a language model in 64 bits, from their definitions: embedding, layer norm, the vocabulary's cross entropy.

Arrays of numpy throughout; 16-bit inputs come as the float64 values that they hold.
"""
from __future__ import annotations

import numpy as np


def embed(tokens, table, scale=1.0):
    out = np.zeros((len(tokens), table.shape[1]))
    for i, t in enumerate(tokens):
        if 0 <= t < table.shape[0]:
            out[i] = scale * table[t]
    return out


def embed_grad(tokens, grad, vocab, scale=1.0, onto=None):
    """(gradient of the table, sum of the magnitudes of what was added, how many)."""
    out = np.zeros((vocab, grad.shape[1])) if onto is None else np.array(onto, np.float64)
    mag, many = np.abs(out), np.zeros(vocab)
    for i, t in enumerate(tokens):
        if 0 <= t < vocab:
            out[t] += scale * grad[i]
            mag[t] += abs(scale) * np.abs(grad[i])
            many[t] += 1
    return out, mag, many


def layer_norm(x, eps):
    """(h, 1 / deviation) of rows."""
    d = x - x.mean(1, keepdims=True)
    r = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    return d * r, r


def layer_norm_grad(x, dy, w, eps):
    h, r = layer_norm(x, eps)
    g = dy * w
    dx = r * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def vocab_loss(x, w, targets, row_weight=None, scale=1.0, c=1.0):
    """{"logp", "loss", "sums", "dz" (scale and c included), "p", "grad_hidden", "grad_weight"}."""
    n, v = x.shape[0], w.shape[0]
    rw = np.ones(n) if row_weight is None else np.asarray(row_weight, np.float64)
    on = np.array([0 <= t < v and q != 0 for t, q in zip(targets, rw)], bool)
    at = np.nonzero(on)[0]
    t = np.asarray(targets)[at]
    z = c * (x[at] @ w.T)
    e = np.exp(z - z.max(1, keepdims=True)) if len(at) else z
    s = e.sum(1, keepdims=True)
    logp = np.zeros(n)
    logp[at] = (z[np.arange(len(at)), t] - z.max(1) - np.log(s[:, 0])) if len(at) else 0
    loss = -rw * logp * on
    p = np.zeros((n, v))
    p[at] = e / s
    dz = p * (scale * c * rw)[:, None]
    dz[at, t] -= scale * c * rw[at]
    xs = np.where(on[:, None], x, 0.0)
    return {"logp": logp, "loss": loss, "sums": np.array([loss.sum(), (rw * on).sum()]), "dz": dz, "p": p, "grad_hidden": dz @ w, "grad_weight": dz.T @ xs}
