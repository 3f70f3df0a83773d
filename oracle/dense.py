"""Plain float64 oracle of the dense layers and of gradient clipping.

TEST INFRASTRUCTURE ONLY, like the rest of ``oracle/``: numpy in float64, from
the definitions alone.

  dense: y = act(x w + b) + r;  dz = dy act'(x w + b), dx = dz w^T, dw = x^T dz,
         db = the sum of dz over the rows
  glu:   [g | u] = x w + b, y = act(g) u;  dz = [dy u act'(g) | dy act(g)]
  clip:  norm = sqrt(sum g^2), each gradient times min(1, max_norm / norm)

relu(z) = max(0, z) with slope [z > 0]; silu(z) = z / (1 + e^-z); gelu(z) =
z Phi(z), Phi the normal distribution function.
"""
from __future__ import annotations

import math

import numpy as np

ACTS = ("none", "relu", "silu", "gelu")
_erf = np.vectorize(math.erf, otypes=[np.float64])


def act(z, name):
    z = np.asarray(z, np.float64)
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    return z


def slope(z, name):
    z = np.asarray(z, np.float64)
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    if name == "gelu":
        phi = np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * phi
    return np.ones_like(z)


def product(x, w, b=None):
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64)
    return z if b is None else z + np.asarray(b, np.float64)


def dense_fwd(x, w, b=None, res=None, name="none"):
    """(y, z)."""
    z = product(x, w, b)
    y = act(z, name)
    return (y if res is None else y + np.asarray(res, np.float64)), z


def dense_dz(dy, z, name):
    return np.asarray(dy, np.float64) * slope(z, name)


def glu_fwd(x, w, b=None, name="silu"):
    """(y, z), z = [g | u]."""
    z = product(x, w, b)
    n = z.shape[1] // 2
    return act(z[:, :n], name) * z[:, n:], z


def glu_dz(dy, z, name):
    n = z.shape[1] // 2
    dy = np.asarray(dy, np.float64)
    return np.concatenate([dy * z[:, n:] * slope(z[:, :n], name), dy * act(z[:, :n], name)], 1)


def layer_bwd(x, w, dz):
    """(dx, dw, db) for the gradient dz of x w + b."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    return dz @ w.T, x.T @ dz, dz.sum(axis=0)


def grad_norm(grads):
    return math.sqrt(sum(float(np.square(np.asarray(g, np.float64)).sum()) for g in grads))


def grad_clip(grads, max_norm):
    """(norm, clipped gradients)."""
    n = grad_norm(grads)
    c = 1.0 if n <= max_norm else max_norm / n
    return n, [np.asarray(g, np.float64) * c for g in grads]
