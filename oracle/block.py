"""Block-sparse attention and the norm and rotation of queries and keys in
fp64 (test infrastructure; shares no code with the GPU path)."""
from __future__ import annotations

import math

import numpy as np


def norm_rope(x, gain, eps, table=None, pos=None, halves=False):
    """x float64 [n][heads][d]; table float [n_pos][d_rot/2][2] of (cos, sin).
    Every row is computed, whatever its position (pos clipped into the table)."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        y = y * np.asarray(gain, np.float64)
    if table is None:
        return y
    t = np.asarray(table, np.float64)
    rows = np.arange(x.shape[0]) if pos is None else np.clip(pos, 0, t.shape[0] - 1)
    f = (t[rows, :, 0] + 1j * t[rows, :, 1])[:, None]
    half = t.shape[1]
    a = np.arange(half) if halves else 2 * np.arange(half)
    b = a + half if halves else a + 1
    z = (y[..., a] + 1j * y[..., b]) * f
    y[..., a], y[..., b] = z.real, z.imag
    return y


def block_means(K, kv_len, block):
    """K [n_obj][n_kv][H_kv][d], kv_len [n_obj] -> [n_obj][H_kv][n_blk][d]."""
    n_obj, n_kv, H_kv, d = K.shape
    nb = -(-n_kv // block)
    out = np.zeros((n_obj, H_kv, nb, d))
    for o in range(n_obj):
        n = min(max(int(kv_len[o]), 0), n_kv)
        for b in range(-(-n // block)):
            out[o, :, b] = K[o, b * block:min((b + 1) * block, n)].mean(0)
    return out


def block_select(Q, Kmean, n_vis, block, top_k, n_first, n_last, n_kv):
    """Q [n_obj][n_q][H][d], Kmean [n_obj][H_kv][n_blk][d] -> idx (filled with
    -1), count."""
    n_obj, n_q, H, _ = Q.shape
    H_kv = Kmean.shape[1]
    idx = np.full((n_obj, n_q, H_kv, top_k), -1, np.int32)
    count = np.zeros((n_obj, n_q, H_kv), np.int32)
    for o in range(n_obj):
        for i in range(n_q):
            nb = -(-min(max(int(n_vis[o, i]), 0), n_kv) // block)
            forced = [b for b in range(nb) if b < n_first or b >= nb - n_last]
            for g in range(H_kv):
                q = Q[o, i].reshape(H_kv, H // H_kv, -1)[g]
                with np.errstate(all="ignore"):
                    s = (Kmean[o, g, :nb] * q[:, None]).sum((0, 2)) if nb else np.zeros(0)
                s = np.where(np.isnan(s), -np.inf, s)
                free = [b for b in np.argsort(-s, kind="stable") if b not in forced]
                keep = sorted(forced + free[:max(0, min(top_k, nb) - len(forced))])
                idx[o, i, g, :len(keep)] = keep
                count[o, i, g] = len(keep)
    return idx, count


def valid_blocks(idx, count, n_blk):
    """The entries of one list that take part (an ascending list has no more than n_blk)."""
    c = min(max(int(count), 0), len(idx), n_blk)
    return [int(b) for t, b in enumerate(idx[:c]) if 0 <= b < n_blk and (t == 0 or b > idx[t - 1])]


def block_attend(Q, K, V, idx, count, n_vis, block):
    """Returns O and the sum of the weights times |V| (for error bounds), both
    [n_obj][n_q][H][d], and the largest sum of |q_c k_c| / sqrt(d) of a row."""
    n_obj, n_q, H, d = Q.shape
    n_kv, H_kv = K.shape[1], K.shape[2]
    nb, G = -(-n_kv // block), H // H_kv
    O, A, L = np.zeros(Q.shape), np.zeros(Q.shape), np.zeros((n_obj, n_q, H, 1))
    for o in range(n_obj):
        for i in range(n_q):
            v = min(max(int(n_vis[o, i]), 0), n_kv)
            for g in range(H_kv):
                js = [np.arange(b * block, min((b + 1) * block, v)) for b in valid_blocks(idx[o, i, g], count[o, i, g], nb)]
                js = np.concatenate(js) if js else np.zeros(0, np.int64)
                if len(js) == 0:
                    continue
                k, w, hs = K[o, js, g], V[o, js, g], slice(g * G, (g + 1) * G)
                z = Q[o, i, hs] @ k.T / math.sqrt(d)
                m = z.max(-1, keepdims=True)
                p = np.exp(z - np.where(np.isfinite(m), m, 0.0))
                t = p.sum(-1, keepdims=True)
                p = p / np.where(t == 0, 1.0, t)
                O[o, i, hs], A[o, i, hs] = p @ w, p @ np.abs(w)
                L[o, i, hs, 0] = (np.abs(Q[o, i, hs]) @ np.abs(k).T).max(-1) / math.sqrt(d)
    return O, A, L
