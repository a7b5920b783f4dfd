"""CPU oracle of the operators around the compressor step: the linear layer, dropout and the random mask, in fp64 numpy,
written from the formulas.  Test infrastructure; it shares no code with the library.

Generator: Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
"""
from __future__ import annotations

import math

import numpy as np

MASK = 0xFFFFFFFF


def philox4x32(counter, key):
    """One call with Python integers: four counter words, two key words -> four words."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK, (a >> 32) ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def philox_words(c0, c1, seed, offset):
    """[len, 4] words (uint64) of counters (c0[i], c1[i], offset low, offset high)."""
    u = np.uint64
    c = [np.asarray(c0, dtype=u), np.asarray(c1, dtype=u)]
    c += [np.full_like(c[0], offset & MASK), np.full_like(c[0], (offset >> 32) & MASK)]
    k = [seed & MASK, (seed >> 32) & MASK]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & u(MASK), (a >> u(32)) ^ c[3] ^ u(k[1]), a & u(MASK)]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return np.stack(c, axis=-1)


def drop_steps(p):
    """p as a multiple of 2^-16."""
    return int(math.floor(p * 65536 + 0.5))


def drop_factor(rows, cols, p, seed=0, offset=0, first_row=0):
    """[rows, cols]: 0 where dropped, 1 / (1 - p) elsewhere; rows first_row ... of a longer array."""
    d = drop_steps(p)
    if d == 0:
        return np.ones((rows, cols))
    groups = (cols + 7) // 8
    w = philox_words(np.tile(np.arange(groups), rows), np.repeat(np.arange(first_row, first_row + rows), groups), seed, offset)
    halves = np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=-1).reshape(rows, groups * 8)[:, :cols]
    return np.where(halves < d, 0.0, 65536.0 / (65536.0 - d) if d < 65536 else 0.0)


def dropout(x, factor, residual=None):
    y = np.where(factor == 0, 0.0, np.where(factor == 0, 0.0, x) * factor)
    return y if residual is None else residual + y


_erf = np.vectorize(math.erf, otypes=[float])


def act(z, kind):
    if kind == "relu":
        return np.where(z < 0, 0.0, z)
    if kind == "gelu":
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if kind == "silu":
        return z / (1 + np.exp(-z))
    return z


def act_slope(z, kind):
    if kind == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if kind == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        t = np.tanh(a * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    return np.ones_like(z)


def linear_forward(x, W, b, kind="identity", factor=None, residual=None):
    """(y, z) with z = x W^T + b, y = residual + D(act(z))."""
    z = x @ W.T
    if b is not None:
        z = z + b
    y = act(z, kind)
    if factor is not None:
        y = dropout(y, factor)
    return (y if residual is None else residual + y), z


def linear_backward(x, W, z, dy, kind="identity", factor=None):
    """(dx, dW, db, dz)."""
    dz = dy if kind == "identity" else dy * act_slope(z, kind)
    if factor is not None:
        dz = dropout(dz, factor)
    return dz @ W, dz.T @ x, dz.sum(0), dz


def mask_keep(n, m, tensor, keep, kept, seed, offset):
    """[n, m] truth values; keep < 0: `kept` of the entries in expectation."""
    below = (kept << 32) // (n * m) if keep < 0 else int(math.floor(keep * 2.0 ** 32 + 0.5))
    c0 = np.arange((n * m + 3) // 4)
    w = philox_words(c0, np.full_like(c0, tensor), seed, offset).reshape(-1)[:n * m]
    return (w < np.uint64(below)).reshape(n, m)


def random_mask_step(grads, errs, keeps):
    """grads[w][t], errs[w][t], keeps[t] (None for vectors) -> (out[t], err[w][t])."""
    W, out, new = len(grads), [], [[] for _ in grads]
    for t, keep in enumerate(keeps):
        if keep is None:
            out.append(sum(g[t].astype(np.float64) for g in grads) / W)
            for e in new:
                e.append(None)
            continue
        M = [grads[w][t].astype(np.float64) + errs[w][t] for w in range(W)]
        out.append(np.where(keep, sum(M) / W, 0.0))
        for w in range(W):
            new[w].append(M[w] - out[-1])
    return out, new
