"""Float64 CPU oracles of include/kv.h, written from the definitions in that header: plain loops over tokens, heads and
pairs where they are cheap, nothing tiled, split or fused.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def pairs_of(rot, interleaved):
    """[(i, j)] of the rotated features, in the order of the table."""
    return [(2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2) for f in range(rot // 2)]


def rotate(y, table, pos, rot, interleaved, sign=1.0):
    """y [T, H, d] turned by R(pos) (sign -1: its transpose)."""
    z = np.array(y, dtype=np.float64)
    for t, p in enumerate(pos):
        for f, (i, j) in enumerate(pairs_of(rot, interleaved)):
            cos, sin = float(table[p, f, 0]), sign * float(table[p, f, 1])
            z[t, :, i] = y[t, :, i] * cos - y[t, :, j] * sin
            z[t, :, j] = y[t, :, j] * cos + y[t, :, i] * sin
    return z


def rms(x, eps):
    return np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def rope_qkv(qkv, Hq, Hkv, wq, wk, eps, table, pos, rot, interleaved):
    """qkv [T, Hq + 2 Hkv, d] -> q, k, v [T, heads, d]."""
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if wq is not None:
        q, k = q / rms(q, eps) * wq, k / rms(k, eps) * wk
    return rotate(q, table, pos, rot, interleaved), rotate(k, table, pos, rot, interleaved), v.copy()


def rope_qkv_bwd(dq, dk, dv, qkv, Hq, Hkv, wq, wk, eps, table, pos, rot, interleaved):
    """Gradients of the packed rows and of the two weights (None without), by the Jacobian of every row."""
    d = qkv.shape[-1]
    out, weights = [], []
    for x, dz, w in ((qkv[:, :Hq], dq, wq), (qkv[:, Hq:Hq + Hkv], dk, wk)):
        g = rotate(dz, table, pos, rot, interleaved, -1.0)
        if w is None:
            out.append(g)
            weights.append(None)
            continue
        n = rms(x, eps)
        dx = np.empty_like(g)
        for t in range(x.shape[0]):
            for h in range(x.shape[1]):
                # d y_j / d x_i = w_j (delta_ij / n - x_i x_j / (d n^3))
                nn, row = n[t, h, 0], x[t, h]
                jac = w[None, :] * (np.eye(d) / nn - np.outer(row, row) / (d * nn ** 3))
                dx[t, h] = jac @ g[t, h]
        out.append(dx)
        weights.append((g * x / n).sum((0, 1)))
    return np.concatenate(out + [dv], 1), weights[0], weights[1]


def decode(q, keys, values, scale):
    """q [Hq, d], keys and values [Hkv, n, d] of one sequence's visible keys -> o [Hq, d], lse [Hq]."""
    Hq, d = q.shape
    G = Hq // keys.shape[0]
    o, lse = np.zeros((Hq, d)), np.full(Hq, -np.inf)
    if keys.shape[1] == 0:
        return o, lse
    for h in range(Hq):
        s = scale * (keys[h // G] @ q[h])
        m = s.max()
        e = np.exp(s - m)
        o[h] = (e[:, None] * values[h // G]).sum(0) / e.sum()
        lse[h] = m + np.log(e.sum())
    return o, lse


def gather(cache, pages, length, page_size):
    """cache [num, Hkv, page_size, d] -> the visible rows [Hkv, n, d] of one sequence (entries outside the cache hide theirs)."""
    rows = [cache[pages[j // page_size], :, j % page_size] for j in range(min(max(length, 0), len(pages) * page_size))
            if 0 <= pages[j // page_size] < cache.shape[0]]
    return np.stack(rows, 1) if rows else np.zeros((cache.shape[1], 0, cache.shape[3]))
