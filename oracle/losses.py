"""Losses of log probabilities with their gradients, and clipping by the norm of all gradients, in float64, as their definitions read.

Rows whose label is outside [0, classes) are masked: no loss, a gradient of zero, and nothing of them is looked at.  A row of minus infinities has no
distribution: no loss, a gradient of zero, but it counts among the unmasked."""
import numpy as np


def log_softmax(x):
    top = np.max(x)
    return x - top - np.log(np.sum(np.exp(x - top)))


def policy_loss(logits, label, old_logp, advantage, clip_low, clip_high, kl_coef, ref_logp=None, ref_logits=None, weight=None):
    """{"loss", "stats": [surrogate, kl, clipped], "logp", "grad"}"""
    x = np.asarray(logits, np.float64)
    rows, C = x.shape
    there = [0 <= a < C for a in label]
    out = {"loss": 0.0, "stats": np.zeros(3), "logp": np.zeros(rows), "grad": np.zeros((rows, C))}
    for r in np.flatnonzero(there):
        a = label[r]
        if np.all(x[r] == -np.inf):
            out["logp"][r] = -np.inf
            continue
        w = float(weight[r]) if weight is not None else 1.0 / sum(there)
        lp = log_softmax(x[r])
        p, onehot, A = np.exp(lp), np.arange(C) == a, float(advantage[r])
        out["logp"][r] = lp[a]
        ratio = np.exp(lp[a] - float(old_logp[r]))
        clipped = (A > 0 and ratio > 1 + clip_high) or (A < 0 and ratio < 1 - clip_low)
        surrogate = A * ((1 + clip_high if A > 0 else 1 - clip_low) if clipped else ratio)
        grad = 0.0 if clipped else -ratio * A * (onehot - p)
        kl = 0.0
        if ref_logp is not None:
            d = float(ref_logp[r]) - lp[a]
            kl = np.expm1(d) - d
            grad = grad - kl_coef * np.expm1(d) * (onehot - p)
        elif ref_logits is not None:
            far = np.zeros(C)
            far[p > 0] = lp[p > 0] - log_softmax(np.asarray(ref_logits[r], np.float64))[p > 0]
            kl = np.sum(p * far)
            grad = grad + kl_coef * p * (far - kl)
        out["loss"] += w * (kl_coef * kl - surrogate)
        out["stats"] += w * np.array([surrogate, kl, float(clipped)])
        out["grad"][r] = w * grad
    return out


def preference_loss(logits, label, offsets, beta, label_smoothing=0.0, ref_logp=None):
    """{"loss", "stats": [mean z, share of z > 0], "logp" of the sequences, "z", "grad"}; rows of no sequence have a gradient of NaN."""
    x = np.asarray(logits, np.float64)
    rows, C = x.shape
    pairs = (len(offsets) - 1) // 2
    L, grad = np.zeros(2 * pairs), np.full((rows, C), np.nan)
    for i in range(2 * pairs):
        for r in range(offsets[i], offsets[i + 1]):
            grad[r] = 0.0
            if 0 <= label[r] < C and not np.all(x[r] == -np.inf):
                lp = log_softmax(x[r])
                L[i] += lp[label[r]]
                grad[r] = (np.arange(C) == label[r]) - np.exp(lp)
    far = L - (np.asarray(ref_logp, np.float64) if ref_logp is not None else 0.0)
    z = beta * (far[0::2] - far[1::2])
    sigma = lambda v: 1.0 / (1.0 + np.exp(-v))  # noqa: E731
    loss = np.zeros(pairs)                                     # (what has no weight counts for nothing, were it infinite)
    for share, v in ((1 - label_smoothing, -z), (label_smoothing, z)):
        if share != 0:
            loss += share * np.logaddexp(0, v)
    dz = label_smoothing * sigma(z) - (1 - label_smoothing) * sigma(-z)
    for i in range(2 * pairs):
        grad[offsets[i]:offsets[i + 1]] *= (1 if i % 2 == 0 else -1) * beta * dz[i // 2] / pairs
    return {"loss": loss.mean(), "stats": np.array([z.mean(), np.mean(z > 0)]), "logp": L, "z": z, "grad": grad}


def grad_norm(grads):
    """(norm of all, of each)"""
    each = np.array([np.sqrt(np.sum(np.square(np.asarray(g, np.float64)))) for g in grads])
    return np.sqrt(np.sum(each ** 2)), each


def grad_clip(grads, max_norm):
    norm, each = grad_norm(grads)
    c = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, each, [np.asarray(g, np.float64) * c for g in grads]
