"""fp64 oracle of the output layer's losses (include/kbest_loss.h), written from the definitions.

NumPy, test infrastructure only.  Every row gets a distribution q over the whole vocabulary (its target with smoothed
labels, or its teacher's softmax over the words that count); the loss is the cross entropy with it, or the divergence
from it.  ``bounds`` gives what a float32 computation of the same may be off by, from the number of operations.
"""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np

U = 2.0 ** -24


@dataclass
class Loss:
    used: np.ndarray     # N bool: the row counts
    q: np.ndarray        # N x V
    x: np.ndarray        # N x V: logits / T
    p: np.ndarray        # N x V
    lse: np.ndarray      # N, 0 where not used
    loss: np.ndarray     # N, 0 where not used
    scale: float         # T^2 for a teacher, 1 for targets
    T: float

    def dlogits(self, grad):
        """Gradients of sum(grad * loss) with respect to h W + b."""
        g = np.where(self.used, grad, 0.0)[:, None] * (self.scale / self.T)
        return np.where(self.used[:, None], g * (self.p - self.q), 0.0)


def _softmax_rows(y):
    top = y.max(axis=1, keepdims=True)
    e = np.exp(y - top)
    s = e.sum(axis=1, keepdims=True)
    return e / s, (top + np.log(s))[:, 0]


def _finish(h, W, b, q, used, T, scale):
    h = np.where(used[:, None], h, 0.0)
    x = (h @ W + b) / T
    p, lse = _softmax_rows(x)
    with np.errstate(divide="ignore", invalid="ignore"):
        logp = np.where(np.isneginf(x), -np.inf, x - lse[:, None])
        known = np.where(q > 0, q * np.log(np.where(q > 0, q, 1.0)), 0.0).sum(1) if scale is not None else 0.0
        cross = -np.where(q > 0, q * logp, 0.0).sum(1)
    loss = (known + cross) * (scale or 1.0)
    return Loss(used, q, x, p, np.where(used, lse, 0.0), np.where(used, loss, 0.0), scale or 1.0, T)


def cross_entropy(h, W, b, target, smoothing=0.0) -> Loss:
    N, V = h.shape[0], W.shape[1]
    used = (target >= 0) & (target < V)
    q = np.zeros((N, V))
    q[used] = smoothing / V
    q[used, target[used]] += 1.0 - smoothing
    return _finish(h, W, b, q, used, 1.0, None)


def distill(h, W, b, token, logit, T=1.0) -> Loss:
    N, V = h.shape[0], W.shape[1]
    counts = (token >= 0) & (token < V) & ~np.isneginf(logit)
    used = counts.any(axis=1)
    q = np.zeros((N, V))
    for n in np.nonzero(used)[0]:
        t, y = token[n][counts[n]], logit[n][counts[n]] / T
        e = np.exp(y - y.max())
        np.add.at(q[n], t, e / e.sum())
    return _finish(h, W, b, q, used, T, T * T)


@dataclass
class Bounds:
    lse: np.ndarray
    loss: np.ndarray
    dx: np.ndarray       # of dlogits before they are rounded to the operands' type


def bounds(o: Loss, h, W, b, f32: bool, grad=None, K=1) -> Bounds:
    """Absolute bounds of a float32 computation.

    A logit: H products and the bias in float32, (H + 3) u of sum |h W| + |b| (float32 operands: six times as many
    products, and 2^-23 of it for the pieces' products that are left out), 1 / T two roundings: d.  A row's sum of exponentials: each
    term off by what its exponent is, d and 4 u of |x| + |max| for the exponent in base 2, 2^-22 for exp2, and chains
    of at most V / 4 + 600 additions: lse by d + that + its own two roundings.  The loss: lse, its words' logits
    (d, and K + 4 roundings of sum q |x|), the smoothed part with chains of V / 4 + 600, and the teacher's part
    (softmax and logarithms: (K + 8) u and 2^-21 of sum q (|ln q| + 1)).
    """
    N, H = h.shape
    V = W.shape[1]
    hh = np.where(o.used[:, None], np.abs(h), 0.0)
    bb = np.where(np.isneginf(b), 0.0, np.abs(b))
    size = (hh @ np.abs(W) + bb) / o.T
    d = ((6 * H + 3) * U + 2.0 ** -23 if f32 else (H + 3) * U) * size + 2 * U * size
    dmax = d.max(1)
    xs = np.where(np.isneginf(o.x), 0.0, np.abs(o.x))
    ex = 4 * U * 2 * xs.max(1) + 2.0 ** -22
    chain = (V / 4 + 600) * U
    lse = dmax + ex + chain + 3 * U * (np.abs(o.lse) + xs.max(1) + 1)
    q = o.q
    lnq = np.where(q > 0, np.abs(np.log(np.where(q > 0, q, 1.0))) + 1, 0.0)
    loss = lse + dmax + (K + 8) * U * ((q * xs).sum(1) + np.abs(o.lse)) + chain * (q * xs).sum(1)
    loss = loss + ((K + 8) * U + 2.0 ** -21) * (q * (lnq + xs)).sum(1)
    loss = loss * o.scale + 3 * U * np.abs(o.loss)
    off = lse[:, None] + d + (4 * U * (xs + np.abs(o.lse)[:, None]) + 2.0 ** -22)
    g = np.abs(np.where(o.used, grad if grad is not None else 0.0, 0.0))[:, None] * (o.scale / o.T)
    dx = g * (o.p * (np.exp(off) - 1) + 4 * U * (o.p + q) + ((K + 8) * U + 2.0 ** -21) * q * (o.scale != 1.0 or K > 1))
    dx = dx + g * 2.0 ** -126
    return Bounds(np.where(o.used, lse, 0.0), np.where(o.used, loss, 0.0), np.where(o.used[:, None], dx, 0.0))
