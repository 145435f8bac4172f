"""Plain fp64 statement of the sequence path: norms of heads with rotation, causal attention over packed histories, attention of new
rows over a cache in pages and over their ancestors.  Test infrastructure: loops over users, rows and heads, no tiling."""
import numpy as np


def norm_rotate(x, gamma, positions, rot_dim, interleaved, base, eps):
    """x [rows x heads x d_h] -> y = x / sqrt(mean(x^2) + eps) * gamma, its pairs turned by position * base^(-2 i / rot_dim)."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    out = y.copy()
    for i in range(rot_dim // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot_dim // 2)
        t = np.asarray(positions, np.float64) * float(base) ** (-2.0 * i / rot_dim)
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return out


def attend(q, k, v, sees, scale):
    """q [n x Hq x d], k, v [m x Hkv x d], sees [n x m] -> (out [n x Hq x d], weighted |v|, scores' magnitude): the second is
    sum_j p_j |v_j|, the third the largest sum_d |q_d| |k_jd| scale of a visible key, both for error bounds.  A key that a row does not
    see is not read for it."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    out, mag, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    G = q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        kh, vh = k[:, h // G], v[:, h // G]
        for i in range(q.shape[0]):
            at = np.flatnonzero(sees[i])
            if len(at) == 0:
                continue
            s = kh[at] @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mag[i, h] = p @ vh[at], p @ np.abs(vh[at])
            size[i, h] = (np.abs(kh[at]) @ np.abs(q[i, h])).max() * scale
    return out, mag, size


def causal(n, m):
    """Row i of the last n of m rows sees the ones up to itself."""
    return np.arange(m)[None, :] <= np.arange(n)[:, None] + (m - n)


def ancestors(parent):
    """Row i sees itself and the chain of its parents; an entry that is not an earlier row ends the chain."""
    n = len(parent)
    sees = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while True:
            sees[i, j] = True
            if not 0 <= parent[j] < j:
                break
            j = parent[j]
    return sees


def cached_rows(pages, table_row, n):
    """The first n rows of a user; pages [P x rows x Hkv x d]; a page that is not there reads as zeros."""
    rows = pages.shape[1]
    out = np.zeros((n,) + pages.shape[2:], np.float64)
    for j in range(n):
        p = table_row[j // rows]
        if 0 <= p < pages.shape[0]:
            out[j] = pages[p, j % rows]
    return out
