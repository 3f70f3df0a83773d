"""Plain float64 oracle of the row operators: layer norm, dropout from a
counter, the residual step of both, and table rows by id.

TEST INFRASTRUCTURE ONLY, like the rest of ``oracle/``: numpy, from the
definitions alone.

  ln:      z = (x - mean) / sqrt(var + eps), y = z gamma + beta (biased variance)
           g = dy gamma, dx = r (g - mean(g) - z mean(g z)), dgamma = sum dy z,
           dbeta = sum dy
  drop:    y = x / q where the value's number is below T, else 0; q = T / 2^32
  drop_ln: h = res + drop(x), y = ln(h); dres = dh + ln's dx, dx = drop(dres)
  embed:   y[r] = scale table[id[r]]; dtable[v] = scale sum of dy[r] with id[r] = v
"""
from __future__ import annotations

import numpy as np

M0, M1 = 0xD2511F53, 0xCD9E8D57
W0, W1 = 0x9E3779B9, 0xBB67AE85
LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=10):
    """Philox4x32 (Salmon, Moraes, Dror and Shaw, SC 2011) on counters [..., 4]
    under one key of two words: the words [..., 4]."""
    c = [np.asarray(counter, np.uint64)[..., i] for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & LOW,
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + W0) & 0xFFFFFFFF, (k[1] + W1) & 0xFFFFFFFF]
    return np.stack(c, -1)


def numbers(rows, c, seed, step, site):
    """The 32-bit number of each value."""
    groups = -(-c // 8)
    i = np.arange(rows * groups, dtype=np.uint64)
    key = (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF)
    out = 0
    for mark, shift in ((0, 16), (1 << 31, 0)):
        ctr = np.empty((rows * groups, 4), np.uint64)
        ctr[:, 0] = i & LOW
        ctr[:, 1] = (i >> np.uint64(32)) + np.uint64((site << 16) + mark)
        ctr[:, 2] = step & 0xFFFFFFFF
        ctr[:, 3] = step >> 32 & 0xFFFFFFFF
        w = philox(ctr, key)
        halves = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1)
        out = out + (halves << np.uint64(shift))
    return out.reshape(rows, groups * 8)[:, :c]


def threshold(p):
    return int(round((1.0 - p) * 2.0 ** 32))


def mask(rows, c, p, seed, step, site=0):
    """(keep, q)."""
    t = threshold(p)
    return numbers(rows, c, seed, step, site) < t, t / 2.0 ** 32


def drop(x, p, seed, step, site=0):
    x = np.asarray(x, np.float64)
    keep, q = mask(*x.shape, p, seed, step, site)
    return np.where(keep, x / q, 0.0)


def stats(x, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    return mean, 1.0 / np.sqrt(np.square(x - mean[:, None]).mean(1) + eps)


def ln_fwd(x, gamma=None, beta=None, eps=1e-5):
    """(y, mean, invstd)."""
    x = np.asarray(x, np.float64)
    mean, r = stats(x, eps)
    y = (x - mean[:, None]) * r[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    return (y if beta is None else y + np.asarray(beta, np.float64)), mean, r


def ln_bwd(x, dy, gamma, invstd):
    """(dx, dgamma, dbeta), the deviations scaled by the given invstd."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    r = np.asarray(invstd, np.float64)[:, None]
    z = (x - x.mean(1, keepdims=True)) * r
    g = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = r * (g - g.mean(1, keepdims=True) - z * (g * z).mean(1, keepdims=True))
    return dx, (dy * z).sum(0), dy.sum(0)


def embed_fwd(ids, table, scale=1.0):
    table = np.asarray(table, np.float64)
    ids = np.asarray(ids, np.int64)
    y = np.zeros((ids.size, table.shape[1]))
    there = (ids >= 0) & (ids < table.shape[0])
    y[there] = table[ids[there]] * scale
    return y


def embed_bwd(ids, dy, num, scale=1.0):
    dy = np.asarray(dy, np.float64)
    ids = np.asarray(ids, np.int64)
    out = np.zeros((num, dy.shape[1]))
    there = (ids >= 0) & (ids < num)
    np.add.at(out, ids[there], dy[there])
    return out * scale
