"""Reference drafted trees over the paged cache, and rotation by positions on several axes.

Test infrastructure; see oracle/__init__.py.  fp64, one node and one head at a time.
"""
import numpy as np

from . import attn
from . import cache


def rotate(x, positions, freq, axis=None, inverse=False):
    """x [T, d] turned by positions [axes, T]; an axis outside the axes leaves its pair."""
    h = x.shape[1] // 2
    y = x.astype(np.float64).copy()
    for i in range(h):
        a = 0 if axis is None else int(axis[i])
        if not 0 <= a < positions.shape[0]:
            continue
        ang = positions[a].astype(np.float64) * float(freq[i]) * (-1 if inverse else 1)
        c, s = np.cos(ang), np.sin(ang)
        y[:, i], y[:, h + i] = x[:, i] * c - x[:, h + i] * s, x[:, h + i] * c + x[:, i] * s
    return y


def ancestors(parents):
    """Of each node: itself, its parent, and so on."""
    up = []
    for t, p in enumerate(parents):
        up.append([t] + (up[p] if 0 <= p < t else []))
    return up


def mask(parents, length, nodes, window=0, sinks=0):
    """(positions [T], sees [T, T] bool) of one tree behind `length` tokens."""
    T = len(parents)
    up = ancestors(parents)
    at = np.array([length + len(up[t]) - 1 if t < nodes else length for t in range(T)], np.int64)
    sees = np.zeros((T, T), bool)
    for t in range(nodes):
        for u in up[t]:
            sees[t, u] = not window or at[t] - at[u] < window or at[u] < sinks
    return at, sees


def words(sees):
    """sees [.., T, T] as int32 words of 32 nodes."""
    T = sees.shape[-1]
    n = (T + 31) // 32
    bits = np.zeros(sees.shape[:-1] + (32 * n,), bool)
    bits[..., :T] = sees
    packed = np.packbits(bits.reshape(bits.shape[:-1] + (n, 4, 8)), axis=-1, bitorder="little")
    return packed.reshape(bits.shape[:-1] + (n, 4)).copy().view("<i4")[..., 0]


def attention(q, k, v, ks, vs, table, lens, sees, at, counts, window, sinks, scale):
    """q [B, Hq, T, d], sees [B, T, T], at [B, T] (used with a window) -> out, its bound, lse.  The bound: half a step of
    8 significant bits for each weight and for the result, and what the weights' smallest step leaves of them."""
    B, Hq, T, d = q.shape
    G = Hq // k.shape[1]
    out, err, lse = np.zeros_like(q), np.zeros_like(q), np.full((B, Hq, T), -np.inf)
    for b in range(B):
        n = int(lens[b])
        m = min(int(counts[b]), n)
        base = n - m
        j = np.arange(n)
        see = np.zeros((T, n), bool)
        for t in range(m):
            p = min(max(int(at[b, t]), base), n - 1) if window else n
            see[t, :base] = (p - j[:base] < window) | (j[:base] < sinks) if window else True
            see[t, base:] = sees[b, t, :m]
        for h in range(Hq):
            if n == 0:
                continue
            kk, vv, have = cache.gather(k, v, ks, vs, table, n, b, h // G)
            seen = attn.seen_keys(see & have[None])
            if seen.size == 0:
                continue
            kx, vx, mx = kk[seen], vv[seen], (see & have[None])[:, seen]
            out[b, h], lse[b, h] = attn.head_fwd(q[b, h], kx, vx, mx, scale)
            p = attn.head_probs(q[b, h], kx, mx, scale)
            err[b, h] = (1 + 2.0 ** -4) * (2.0 ** -8 * np.abs(out[b, h]) + 2.0 ** -8 * (p @ np.abs(vx)))
    return out, err, lse
