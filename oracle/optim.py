"""Global gradient-norm clipping, Adam, RMSprop and Muon, over the flat parameter buffer.

Test infrastructure: only the tests, the smoke check and the benchmark's CPU baseline use
this package.

Algorithm 1 clips the maximum gradient norm of all parameters (policy and value share the
trunk) before the optimiser step; Appendix B sets the threshold (PPO 0.5, IMPALA 40) and
Adam's epsilon (1e-5). beta1 = 0.9, beta2 = 0.999 and bias correction are the standard Adam
(Kingma and Ba, 2015) values, as used by optax. Appendix B's IMPALA table gives RMSprop with
epsilon 0.01 and decay 0.99; where epsilon sits is not stated, and it is read as optax's
RMSprop does it: inside the square root, with the second-moment estimate starting at zero
(the paper's learner is written in JAX). Muon is no part of the paper: it is written from its formulas, the
momentum's orthogonalisation by five steps of a quintic Newton-Schulz iteration.
"""
from __future__ import annotations

import numpy as np


def global_norm(g):
    return float(np.sqrt(np.sum(np.asarray(g, np.float64) ** 2)))


def clip_by_global_norm(g, max_norm, dtype=np.float64):
    """g * (max_norm / ||g||) when ||g|| > max_norm, else g unchanged; max_norm <= 0 disables.
    Returns (clipped g, pre-clip norm)."""
    g = np.asarray(g, dtype)
    n = np.sqrt(np.sum(g * g))
    if max_norm > 0 and n > max_norm:
        g = g * (max_norm / n)
    return g, n


def adam(p, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-5, dtype=np.float64):
    """One Adam update at 1-based ``step``; returns new (p, m, v).

    m <- b1 m + (1-b1) g;  v <- b2 v + (1-b2) g^2
    p <- p - lr * (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
    """
    p, g, m, v = (np.asarray(a, dtype) for a in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mhat = m / (1 - beta1 ** step)
    vhat = v / (1 - beta2 ** step)
    return p - lr * mhat / (np.sqrt(vhat) + eps), m, v


def rmsprop(p, g, nu, lr, decay=0.99, eps=0.01, dtype=np.float64):
    """One RMSprop update; returns new (p, nu).

    nu <- decay nu + (1 - decay) g^2
    p  <- p - lr * g / sqrt(nu + eps)
    """
    p, g, nu = (np.asarray(a, dtype) for a in (p, g, nu))
    nu = decay * nu + (1 - decay) * g * g
    return p - lr * g / np.sqrt(nu + eps), nu


QUINTIC = (3.4445, -4.7750, 2.0315)


def orthogonalize(x, steps=5, eps=1e-7, dtype=np.float64):
    """X0 = x / max(||x||_F, eps), then ``steps`` times X <- a X + b (X X^T) X + c (X X^T)^2 X."""
    x = np.asarray(x, dtype)
    X = x / max(np.sqrt(np.sum(x * x)), eps)
    a, b, c = (dtype(k) for k in QUINTIC)
    for _ in range(steps):
        if X.shape[0] <= X.shape[1]:
            A = X @ X.T
            X = a * X + (b * A + c * (A @ A)) @ X
        else:
            A = X.T @ X
            X = a * X + X @ (b * A + c * (A @ A))
    return X


def muon(p, g, m, v, step, mats, lr, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, scale=0, eps=1e-7,
         adam_lr=2.5e-4, beta1=0.9, beta2=0.999, adam_eps=1e-5, dtype=np.float64):
    """One Muon update; returns new (p, m, v). For every (offset, rows, cols) of ``mats``:

    m <- mu m + (1 - mu) g;  u = mu m + (1 - mu) g if nesterov else m
    p <- p (1 - lr weight_decay) - lr s O(u), s = sqrt(max(1, cols / rows)), or 0.2 sqrt(max(rows, cols)) for scale 1
    (v is left alone there); Adam with adam_lr on everything else.
    """
    p, g, m, v = (np.asarray(a, dtype) for a in (p, g, m, v))
    p1, m1, v1 = adam(p, g, m, v, step, adam_lr, beta1, beta2, adam_eps, dtype)
    for off, rows, cols in mats:
        at = slice(off, off + rows * cols)
        m1[at] = momentum * m[at] + (1 - momentum) * g[at]
        u = momentum * m1[at] + (1 - momentum) * g[at] if nesterov else m1[at]
        s = np.sqrt(max(1.0, cols / rows)) if scale == 0 else 0.2 * np.sqrt(max(rows, cols))
        O = orthogonalize(u.reshape(rows, cols), steps, eps, dtype)
        p1[at] = p[at] * (1 - lr * weight_decay) - lr * s * O.ravel()
        v1[at] = v[at]
    return p1, m1, v1
