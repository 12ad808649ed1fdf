"""Oracle distillation from a teacher's top logits, with gradients.

TEST INFRASTRUCTURE ONLY (see the package docstring).

The teacher's probabilities are laid out over the whole vocabulary (entries with a
negative id are not there; the same id more than once adds up), and everything follows
from loss_r = weight_r sum_j p_j (log p_j - log q(ids_j)).
"""
from __future__ import annotations

import numpy as np


def teacher(ids, logits, teacher_scale=1.0, t_lse=None):
    """p [rows, k] of the entries (0 where there is none) and their log-probabilities."""
    t = np.where(ids >= 0, logits * teacher_scale, -np.inf)
    if t_lse is None:
        top = t.max(1, keepdims=True)
        top = np.where(np.isfinite(top), top, 0.0)
        s = np.exp(t - top).sum(1, keepdims=True)
        with np.errstate(divide="ignore"):
            norm = top + np.log(s)
    else:
        norm = t_lse[:, None]
    with np.errstate(invalid="ignore"):
        logp = np.where(t == -np.inf, -np.inf, t - norm)
    return np.exp(logp), logp


def loss_and_grads(h, w, ids, logits, logit_scale=1.0, teacher_scale=1.0, loss_scale=1.0, t_lse=None, weight=None):
    """h [rows, H], w [V, H] float64 -> dict(loss_tok, lse, loss_sum, dh, dw, dz)."""
    rows = len(h)
    weight = np.ones(rows) if weight is None else weight
    z = logit_scale * (h @ w.T)
    top = z.max(1, keepdims=True)
    lse = top + np.log(np.exp(z - top).sum(1, keepdims=True))
    p, logp = teacher(ids, logits, teacher_scale, t_lse)
    at = np.maximum(ids, 0)
    with np.errstate(invalid="ignore"):
        term = np.where(p > 0, p * (logp - np.take_along_axis(z, at, 1) + lse), 0.0)
    loss = weight * term.sum(1)
    dense = np.zeros_like(z)
    for r in range(rows):
        np.add.at(dense[r], at[r], np.where(ids[r] >= 0, p[r], 0.0))
    g = (loss_scale * weight)[:, None]
    dz = g * (np.exp(z - lse) * p.sum(1, keepdims=True) - dense)
    return dict(loss_tok=loss, lse=lse[:, 0], loss_sum=loss_scale * loss.sum(), dz=dz, z=z, p=p,
                dh=logit_scale * (dz @ w), dw=logit_scale * (dz.T @ h))
