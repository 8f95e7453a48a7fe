"""The operators of the training step in 64 bits, from their definitions: policy loss, gradient norm, clipping, AdamW.

Arrays of numpy throughout; 16-bit inputs come as the float64 values that they hold.
"""
from __future__ import annotations

import numpy as np

SUMS = ("loss", "pg", "kl", "clipped", "weight")


def policy_loss(z, targets, old=None, ref=None, adv=None, weight=None, scale=1.0, clip_low=0.2, clip_high=0.2, kl_coef=0.0, c=1.0):
    """{"logp", "loss", "sums", "grad"} of rows of logits z (c = 1 / temperature)."""
    z = np.asarray(z, np.float64)
    rows, vocab = z.shape
    w = np.ones(rows) if weight is None else np.asarray(weight, np.float64)
    logp, loss, grad, sums = np.zeros(rows), np.zeros(rows), np.zeros((rows, vocab)), np.zeros(5)
    for i in range(rows):
        t = int(targets[i])
        if w[i] == 0 or not 0 <= t < vocab or np.all(z[i] == -np.inf):
            continue
        with np.errstate(all="ignore"):
            e = np.exp(c * (z[i] - z[i].max()))
            p = e / e.sum()
            logp[i] = c * (z[i, t] - z[i].max()) - np.log(e.sum())
            if adv is None:
                continue
            a = float(adv[i])
            r = 1.0 if old is None else np.exp(logp[i] - float(old[i]))
            if a >= 0:
                used, clipped = min(r, 1.0 + clip_high), r > 1.0 + clip_high
            else:
                used, clipped = max(r, 1.0 - clip_low), r < 1.0 - clip_low
            used = r if np.isnan(r) else used
            pg, slope = -a * used, 0.0 if clipped else -a * r
            kl, value = 0.0, pg
            if ref is not None:
                d = float(ref[i]) - logp[i]
                kl = np.inf if d == np.inf else np.expm1(d) - d
                if kl_coef != 0:            # (an infinite penalty that is only watched is not part of the loss)
                    slope -= kl_coef * np.expm1(d)
                    value = pg + kl_coef * kl
            loss[i] = w[i] * value
            sums += np.array([loss[i], w[i] * pg, w[i] * kl, w[i] * clipped, w[i]])
            onehot = np.zeros(vocab)
            onehot[t] = 1.0
            grad[i] = scale * w[i] * slope * c * (onehot - p)
    return {"logp": logp, "loss": loss, "sums": sums, "grad": grad}


def grad_norm(tensors, kind="2", scale=1.0):
    flat = np.concatenate([np.asarray(t, np.float64).ravel() for t in tensors]) if tensors else np.zeros(0)
    if flat.size == 0:
        return 0.0
    return abs(scale) * (np.sqrt(np.sum(flat * flat)) if kind == "2" else np.max(np.abs(flat)))


def clip_factor(norm, max_norm, scale=1.0):
    q = max_norm / (norm + 1e-6)
    return scale * (1.0 if q > 1.0 else q)


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, factor=1.0):
    """(p, m, v) behind one update by the gradient g * factor."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    h = g * factor
    m = beta1 * m + (1.0 - beta1) * h
    v = beta2 * v + (1.0 - beta2) * h * h
    p = p - lr * weight_decay * p - lr * (m / (1.0 - beta1 ** step)) / (np.sqrt(v / (1.0 - beta2 ** step)) + eps)
    return p, m, v
