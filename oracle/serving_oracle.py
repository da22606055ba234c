"""Plain fp64 numpy statements of the serving calls (rbs_paged_extend, rbs_qk_norm_rope, rbs_qk_norm_rope_paged,
rbs_paged_decode), written from the formulas in include/rbs.h.  Slow on purpose; shares no code with the CUDA path."""
from __future__ import annotations

import numpy as np


def extend(seq_lens, new_lens, table, free_pages, page, n_pages, n_tokens, used=0):
    """Token by token: a token that begins a page takes the next free one.  Returns (table, lens, cu, positions, slots, used)."""
    table = np.array(table)
    cap = table.shape[1] * page
    positions, slots = np.zeros(n_tokens, np.int64), np.full(n_tokens, -1, np.int64)
    lens, cu, row = [], [0], 0
    for s, (have, new) in enumerate(zip(seq_lens, new_lens)):
        n = min(max(int(have), 0), cap)
        end = n
        for _ in range(min(max(int(new), 0), n_tokens - row)):
            positions[row] = end
            if end < cap:
                if end % page == 0:
                    table[s, end // page] = free_pages[used] if used < len(free_pages) else -1
                    used += 1
                p = int(table[s, end // page])
                if 0 <= p < n_pages:
                    slots[row] = p * page + end % page
            end += 1
            row += 1
        lens.append(min(end, cap))
        cu.append(row)
    return table, np.array(lens), np.array(cu), positions, slots, used


def norm_rope(x, positions, inv_freq, weight=None, eps=1e-6, interleaved=False, magnitude=1.0):
    """x [..., tokens, heads, d] -> (result, size), size = magnitude * (|y_u| + |y_v|) of the pair behind each element (|y| outside)."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    out, size = y.copy(), np.abs(y)
    n = len(inv_freq)
    for i in range(n):
        u, v = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        a = (np.asarray(positions, np.float64) * np.float64(inv_freq[i]))[:, None]
        out[..., u] = magnitude * (y[..., u] * np.cos(a) - y[..., v] * np.sin(a))
        out[..., v] = magnitude * (y[..., v] * np.cos(a) + y[..., u] * np.sin(a))
        size[..., u] = size[..., v] = abs(magnitude) * (np.abs(y[..., u]) + np.abs(y[..., v]))
    return out, size


def decode(q, k_cache, v_cache, table, lens, scale=None):
    """q [S, Hq, d], caches [pages, page, Hkv, d].  Returns (out, lse, size): size = sum of softmax * |v|."""
    S, Hq, d = q.shape
    n_pages, page, Hkv, _ = k_cache.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, size, lse = np.zeros((S, Hq, d)), np.zeros((S, Hq, d)), np.full((S, Hq), -np.inf)
    for s in range(S):
        at = [(int(table[s, t // page]), t % page) for t in range(min(max(int(lens[s]), 0), table.shape[1] * page))]
        at = [(p, o) for p, o in at if 0 <= p < n_pages]
        if not at:
            continue
        pages, offs = np.array([p for p, _ in at]), np.array([o for _, o in at])
        for h in range(Hq):
            hk = h // (Hq // Hkv)
            k, v = (np.asarray(c[pages, offs, hk], np.float64) for c in (k_cache, v_cache))
            x = scale * (k @ np.asarray(q[s, h], np.float64))
            top = x.max()
            e = np.exp(x - top)
            lse[s, h] = top + np.log(e.sum())
            out[s, h] = e @ v / e.sum()
            size[s, h] = e @ np.abs(v) / e.sum()
    return out, lse, size
