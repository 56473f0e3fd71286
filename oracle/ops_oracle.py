"""fp64 CPU reference of the operators around the loss (test infrastructure
only): top-K entries, the teacher cache, 8-bit checkpoints and draft
verification, each written from its definition in NumPy."""
from __future__ import annotations

import numpy as np

CODE_MAX = 4094
REACH = 1024.0
FLT_MAX = float(np.finfo(np.float32).max)


def topk_entries(logits, K, logprobs=False):
    """(index [N, K], value [N, K]) of the K largest logits: a number that is
    none counts as -inf; equal ones in index order. Log-probabilities: z minus
    the log of the sum of exp over the row."""
    z = np.array(logits, dtype=np.float64)
    z[np.isnan(z)] = -np.inf
    z += 0.0
    idx = np.argsort(-z, axis=1, kind="stable")[:, :K]
    val = np.take_along_axis(z, idx, 1)
    if not logprobs:
        return idx, val
    out = np.full_like(val, -np.inf)
    for n in range(z.shape[0]):
        m = z[n].max()
        if m == -np.inf:
            continue
        with np.errstate(invalid="ignore"):  # inf - inf, not taken
            d = np.where(z[n] == m, 0.0, z[n] - m)
            dv = np.where(val[n] == m, 0.0, val[n] - m)
        out[n] = dv - np.log(np.exp(d).sum())
    return idx, out


def cache_write(logits, K, logprobs=False):
    """(entries [N, K], top [N] in fp64, step [N] fp32)."""
    idx, val = topk_entries(logits, K)
    _, out = topk_entries(logits, K, logprobs)
    N = idx.shape[0]
    entries = np.zeros((N, K), dtype=np.int64)
    top, step = np.full(N, -np.inf), np.zeros(N, dtype=np.float32)
    for n in range(N):
        if val[n, 0] == -np.inf:
            entries[n] = idx[n] << 12 | 4095
            continue
        v = np.minimum(val[n], FLT_MAX)
        kept = v >= v[0] - REACH
        step[n] = np.float32((v[0] - v[kept].min()) / CODE_MAX)
        s = float(step[n])
        code = np.full(K, 4095, dtype=np.int64)
        code[kept] = np.minimum(np.rint((v[0] - v[kept]) / s), CODE_MAX) if s > 0 else 0
        entries[n] = idx[n] << 12 | code
        top[n] = out[n, 0] if logprobs else v[0]
    return entries, top, step


def cache_read(entries, scale, rows=None):
    """(teacher_idx, teacher_logit, ignore) of cache rows."""
    e = np.asarray(entries).astype(np.int64) & 0xffffffff
    sc = np.asarray(scale, dtype=np.float64)
    N, K = e.shape
    rows = np.arange(N) if rows is None else np.asarray(rows)
    idx = np.full((len(rows), K), -1, dtype=np.int64)
    logit = np.zeros((len(rows), K))
    ignore = np.ones(len(rows), dtype=np.uint8)
    for m, r in enumerate(rows):
        if r < 0 or r >= N or sc[r, 0] == -np.inf:
            continue
        ignore[m] = 0
        idx[m] = e[r] >> 12
        code = e[r] & 4095
        logit[m] = np.where(code == 4095, -np.inf, sc[r, 0] - code * sc[r, 1])
    return idx, logit, ignore


def checkpoint(hidden):
    """(values, scale bytes) of 8-bit checkpoints: blocks of 32 columns, the
    nearest value of 4 significant bits (ties to even; multiples of 2^-9 below
    2^-6) of each element over the block's power of two."""
    x = np.asarray(hidden, dtype=np.float64)
    b = x.reshape(x.shape[0], -1, 32)
    out = np.empty_like(b)
    s = np.zeros(b.shape[:2], dtype=np.int64)
    for n in range(b.shape[0]):
        for j in range(b.shape[1]):
            v = b[n, j]
            if not np.isfinite(v).all():
                s[n, j] = 255
                out[n, j] = np.nan
                continue
            a = np.abs(v).max()
            e = -127
            while e < 127 and a > 448.0 * 2.0 ** e:
                e += 1
            s[n, j] = e + 127
            t = v / 2.0 ** e
            _, p = np.frexp(t)
            grid = np.exp2(np.maximum(p - 1, -6) - 3.0)
            # (what would round to 2^128 is held as the value below it)
            out[n, j] = np.clip(np.rint(t / grid) * grid * 2.0 ** e, -1.875 * 2.0 ** 127,
                                1.875 * 2.0 ** 127)
    return out.reshape(x.shape), s


def softmax(z, tau):
    z = np.array(z, dtype=np.float64)
    z[np.isnan(z)] = -np.inf
    m = z.max()
    if m == -np.inf:
        return np.zeros_like(z)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp(np.where(z == m, 0.0, z - m) / tau)
    return w / w.sum()


def draft_distribution(idx, logit, V, tau):
    """Dense [V] distribution of K entries: indices outside [0, V) keep their
    share of the softmax but belong to no token."""
    q = np.zeros(V)
    for v, w in zip(idx, softmax(logit, tau)):
        if 0 <= v < V:
            q[v] += w
    return q


def verify_draft(target, tokens, uniform, q, lengths=None, tau=1.0):
    """One sequence after the other. target [B, T+1, V], q [B, T, V] the draft's
    probabilities. Returns (tokens, accepted, accept_prob)."""
    B, T1, V = target.shape
    T = T1 - 1
    out = np.full((B, T1), -1, dtype=np.int64)
    acc = np.zeros(B, dtype=np.int64)
    prob = np.zeros((B, T))
    for b in range(B):
        n = T if lengths is None else int(min(max(lengths[b], 0), T))
        p = [softmax(target[b, t], tau) for t in range(n + 1)]
        r = n
        for t in range(n):
            d = int(tokens[b, t])
            known = 0 <= d < V
            pd, qd = (p[t][d], q[b, t, d]) if known else (0.0, 0.0)
            prob[b, t] = min(1.0, pd / qd) if qd > 0 else float(pd > 0)
            if r == n and not float(uniform[b, t]) * qd < pd:
                r = min(r, t)
        out[b, :r] = tokens[b, :r]
        acc[b] = r
        x = p[r]
        if r < n:
            rest = np.maximum(p[r] - q[b, r], 0.0)
            x = rest if rest.sum() > 0 else x
        if x.sum() > 0:
            c = np.cumsum(x)
            v = int(np.searchsorted(c, float(uniform[b, T]) * c[-1], side="right"))
            out[b, r] = min(v, int(np.nonzero(x)[0][-1]))
    return out, acc, prob
