"""The paged key/value cache in float64 NumPy, row by row from the formulas.

A pool is [pages, page_size, 2 kvd]; row r of sequence b is row r % page_size
of page table[b][r // page_size]. A page id outside the pool reads as zeros and
loses what is stored there.
"""
import numpy as np


def rows(pool, ids, n):
    """The first n rows behind a list of page ids."""
    size = pool.shape[1]
    out = np.zeros((n, pool.shape[2]))
    for r in range(n):
        page = int(ids[r // size])
        if 0 <= page < pool.shape[0]:
            out[r] = pool[page, r % size]
    return out


def rotate(x, pos, theta, hd):
    """Every head of x [T, heads * hd]: pairs (i, i + hd/2) by pos theta^(-2i/hd)."""
    z = np.asarray(x, np.float64).reshape(len(x), -1, 2, hd // 2)
    angle = np.asarray(pos, np.float64)[:, None] * float(theta) ** (-2.0 * np.arange(hd // 2) / hd)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    out = np.stack([z[:, :, 0] * c - z[:, :, 1] * s, z[:, :, 1] * c + z[:, :, 0] * s], axis=2)
    return out.reshape(len(x), -1)


def append(pool, table, cu, kv_len, k, v):
    """A copy of the pool with the rows k | v (rotated already) stored."""
    out, size = np.array(pool, np.float64), pool.shape[1]
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        for r in range(n):
            row = int(kv_len[b]) - n + r
            if row < 0 or row // size >= table.shape[1]:
                continue
            page = int(table[b, row // size])
            if 0 <= page < pool.shape[0]:
                out[page, row % size] = np.concatenate([k[cu[b] + r], v[cu[b] + r]])
    return out


def attention(q, pool, table, cu, kv_len, n_heads, n_kv_heads, causal, scale=None, prefix_pages=None,
              prefix_len=0, max_kv_len=None):
    """(out [T, H hd], lse [H, T], and for error bounds sum_j p_j |v_j| as out
    and the largest scale sum |q| |k| of a row as lse)."""
    T, hd = len(q), q.shape[1] // n_heads
    G, kvd = n_heads // n_kv_heads, n_kv_heads * hd
    scale = hd ** -0.5 if scale is None else scale
    most = table.shape[1] * pool.shape[1] if max_kv_len is None else max_kv_len
    out, lse = np.zeros((T, n_heads, hd)), np.full((n_heads, T), -np.inf)
    size, mag = np.zeros((T, n_heads, hd)), np.zeros((n_heads, T))
    head = rows(pool, prefix_pages, prefix_len) if prefix_len else np.zeros((0, 2 * kvd))
    qh = np.asarray(q, np.float64).reshape(T, n_heads, hd)
    for b in range(len(cu) - 1):
        n, m = cu[b + 1] - cu[b], max(0, min(int(kv_len[b]), most))
        kv = np.concatenate([head, rows(pool, table[b], m)]).reshape(-1, 2, n_kv_heads, hd)
        for r in range(n):
            own = min(m, int(kv_len[b]) - n + r + 1) if causal else m
            seen = kv[:prefix_len + max(0, own)]
            t = cu[b] + r
            for h in range(n_heads if len(seen) else 0):
                kk, vv = seen[:, 0, h // G], seen[:, 1, h // G]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = kk @ qh[t, h] * scale
                    p = np.exp(s - s.max())
                    out[t, h] = p @ vv / p.sum()
                    lse[h, t] = s.max() + np.log(p.sum())
                    size[t, h] = p @ np.abs(vv) / p.sum()
                    mag[h, t] = (np.abs(kk) @ np.abs(qh[t, h])).max() * scale
    return out.reshape(T, -1), lse, size.reshape(T, -1), mag
