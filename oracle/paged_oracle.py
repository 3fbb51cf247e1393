"""Plain float64 CPU reference of the operators on a paged latent cache.

TEST INFRASTRUCTURE ONLY: only the test-suite may import it.  It shares no code with the GPU
path and imports nothing from it.

Position p of sequence b lies in row p % page_size of page table[b, p // page_size] of the pool
[n_pages, page_size, width]; a row is [c^KV | R_p k^PE] (Eq. 5's cache).
"""
from __future__ import annotations

import numpy as np


def rotate(x, pos, inv_freq):
    """R_pos x for rotate-half pairs (d, d + n/2): x [..., n], inv_freq [n/2]."""
    half = x.shape[-1] // 2
    z = (x[..., :half] + 1j * x[..., half:]) * np.exp(1j * float(pos) * np.asarray(inv_freq, np.float64))
    return np.concatenate([z.real, z.imag], axis=-1)


def append(pool, table, rows, q, offsets, start, inv_freq, *, kv_rank, nope_dim):
    """(pool, q_out) after the packed rows entered the cache; q_out rows of no sequence are NaN.

    rows [n, kv_rank + G_r dr], q [n, H, nope_dim + dr], inv_freq [G_r, dr / 2]."""
    pool, q_out = pool.copy(), np.full(q.shape, np.nan)
    ps, (Gr, half) = pool.shape[1], inv_freq.shape
    for b in range(len(start)):
        for i in range(int(offsets[b]), int(offsets[b + 1])):
            p = int(start[b]) + i - int(offsets[b])
            if p // ps < table.shape[1] and 0 <= table[b, p // ps] < len(pool):
                row = rows[i].copy()
                for g in range(Gr):
                    c = kv_rank + 2 * half * g
                    row[c:c + 2 * half] = rotate(row[c:c + 2 * half], p, inv_freq[g])
                pool[table[b, p // ps], p % ps] = row
            q_out[i] = q[i]
            for h in range(q.shape[1]):
                g = h // (q.shape[1] // Gr)
                q_out[i, h, nope_dim:] = rotate(q[i, h, nope_dim:], p, inv_freq[g])
    return pool, q_out


def cached_rows(pool, table, b, n):
    """The first n rows of sequence b (NaN where the table names no page)."""
    ps = pool.shape[1]
    out = np.full((n, pool.shape[2]), np.nan)
    for p in range(n):
        page = table[b, p // ps]
        if 0 <= page < len(pool):
            out[p] = pool[page, p % ps]
    return out


def attend(q, rows, Wuk, Wuv, *, nope_dim, scale, n_groups, first):
    """o [t, H, d_v] of query tokens at positions first .. first + t - 1 over the cached rows:
    keys [W_UK c | k^PE] and values W_UV c written out, rows after a token's position unseen."""
    t, H, _ = q.shape
    rkv, dv = Wuk.shape[1], Wuv.shape[0] // n_groups
    out = np.zeros((t, H, dv))
    for h in range(H):
        g = h // (H // n_groups)
        keys = np.concatenate([rows[:, :rkv] @ Wuk[g * nope_dim:(g + 1) * nope_dim].T, rows[:, rkv:]], axis=1)
        values = rows[:, :rkv] @ Wuv[g * dv:(g + 1) * dv].T
        for r in range(t):
            n = min(max(first + r + 1, 0), len(rows))
            if n == 0:
                continue
            s = keys[:n] @ q[r, h] * scale
            p = np.exp(s - s.max())
            out[r, h] = (p / p.sum()) @ values[:n]
    return out
