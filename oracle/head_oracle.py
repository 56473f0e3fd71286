"""fp64 CPU reference of the output head's operators (test infrastructure only):
4-bit microscaled numbers, logits with a head of them, and cross entropy against
labels with its gradients, each written from its definition in NumPy."""
from __future__ import annotations

import math

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_write(x):
    """(codes [N, D / 2] uint8, scales [N, D / 32] uint8): element by element, the
    nearest of the eight magnitudes, of two the one with the even code."""
    x = np.asarray(x, dtype=np.float64)
    N, D = x.shape
    b = x.reshape(N, D // 32, 32)
    scales = np.zeros((N, D // 32), dtype=np.uint8)
    codes = np.zeros((N, D // 32, 32), dtype=np.uint8)
    for n in range(N):
        for j in range(D // 32):
            v = b[n, j]
            if not np.isfinite(v).all():
                scales[n, j] = 255
                continue
            top = np.abs(v).max()
            s = -127
            if top > 0:
                s = max(-127, math.frexp(top / 6.0)[1] - 1)
                while top > math.ldexp(6.0, s):
                    s += 1
                while s > -127 and top <= math.ldexp(6.0, s - 1):
                    s -= 1
            scales[n, j] = s + 127
            t = np.ldexp(np.abs(v), -s)
            if s == 126:
                t = np.minimum(t, 3.0)
            d = np.abs(t[:, None] - VALUES)
            best = d.argmin(axis=1)                       # the lower one of two
            up = np.minimum(best + 1, 7)
            tie = (d[np.arange(32), up] == d[np.arange(32), best]) & (best % 2 == 1)
            c = np.where(tie, up, best)
            codes[n, j] = c + 8 * np.signbit(v)
    c = codes.reshape(N, D)
    return c[:, 0::2] | (c[:, 1::2] << 4), scales


def mx4_read(codes, scales):
    """The values in fp64 (2^128 and more included: infinite in the narrower types)."""
    codes, scales = np.asarray(codes), np.asarray(scales)
    N = codes.shape[0]
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(N, -1)
    v = VALUES[c & 7] * np.where(c >= 8, -1.0, 1.0)
    s = np.repeat(np.ldexp(1.0, scales.astype(np.int64) - 127), 32, axis=1)
    return np.where(np.repeat(scales == 255, 32, axis=1), np.nan, v * s)


def mx4_logits(hidden, codes, scales):
    """(logits, the sums of the products' magnitudes) in fp64."""
    h, w = np.asarray(hidden, dtype=np.float64), mx4_read(codes, scales)
    return h @ w.T, np.abs(h) @ np.abs(w).T


def cross_entropy(hidden, W, labels, z_loss=0.0, g=1.0, g_token=None):
    """Mean over the tokens whose label is in [0, V) of ln Z - z[label] + z_loss
    (ln Z)^2 (0 if there are none), and the gradients of g times it (or of sum_t
    g_token[t] l_t). size: the larger magnitude of ln Z and z[label], whose difference
    the loss is; q_label: the label's probability; weight: of each token."""
    h, W = np.asarray(hidden, dtype=np.float64), np.asarray(W, dtype=np.float64)
    labels = np.asarray(labels)
    N, V = h.shape[0], W.shape[0]
    valid = (labels >= 0) & (labels < V)
    n = int(valid.sum())
    z = h @ W.T
    top = z.max(axis=1, keepdims=True)
    e = np.exp(z - top)
    total = e.sum(axis=1, keepdims=True)
    logz = (np.log(total) + top)[:, 0]
    at = np.where(valid, labels, 0)
    rows = np.arange(N)
    lpt = np.where(valid, logz - z[rows, at] + z_loss * logz ** 2, 0.0)
    weight = np.full(N, g / n if n else 0.0) if g_token is None else np.asarray(g_token, np.float64)
    weight = np.where(valid, weight, 0.0)
    G = e / total * (1.0 + 2.0 * z_loss * logz)[:, None]
    G[rows, at] -= 1.0
    G *= weight[:, None]
    return dict(loss=lpt.sum() / n if n else 0.0, loss_per_token=lpt,
                logz=np.where(valid, logz, 0.0),
                size=np.where(valid, np.maximum(np.abs(logz), np.abs(z[rows, at])), 0.0),
                q_label=np.where(valid, e[rows, at] / total[:, 0], 0.0), weight=weight,
                grad_hidden=G @ W, grad_W=G.T @ h)
