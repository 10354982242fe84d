"""Reference attention with a sliding window and sinks, forward and backward.

Test infrastructure; see oracle/__init__.py.  All arithmetic is fp64.  Row i sees
the keys j <= i with i - j < window (window = 0: all) or j < sinks; formulas as
in oracle/attn.py.  Beside each result stands a bound on what rounding the
weights P and dZ to bf16 (relative error at most u = 2^-8 each, independent of
each other) and the result to bf16 may change, element by element:
  out  |o - o'| <= u |o| + 2 u sum P |v|       (numerator and normaliser)
  dV   u |dV| + u sum P |dO|
  dZ   u |dZ| + P |dO| . err(out)              (Delta is taken from the rounded out)
  dQ   u |dQ| + scale sum err(dZ) |k|,  dK alike
each times 1 + 2^-4 for what the fp32 sums and the exponentials add.
"""
import numpy as np

from . import attn

U = 2.0 ** -8
ROOM = 1 + 2.0 ** -4


def mask(n, window, sinks, first=0):
    """Rows first .. n - 1 against the keys 0 .. n - 1."""
    i, j = np.arange(first, n)[:, None], np.arange(n)[None]
    return (j <= i) & ((i - j < (window or n + 1)) | (j < sinks))


def sequence_fwd(q, k, v, window, sinks, scale):
    """One sequence: q [Hq, n, d], k / v [Hkv, n, d] -> out, its bound, lse, the largest sum |q||k| scale."""
    G = q.shape[0] // k.shape[0]
    m = mask(q.shape[1], window, sinks)
    out, err = np.zeros_like(q), np.zeros_like(q)
    lse = np.zeros(q.shape[:2])
    reach = 0.0
    for h in range(q.shape[0]):
        kk, vv = k[h // G], v[h // G]
        out[h], lse[h] = attn.head_fwd(q[h], kk, vv, m, scale)
        p = attn.head_probs(q[h], kk, m, scale)
        err[h] = ROOM * (U * np.abs(out[h]) + 2 * U * (p @ np.abs(vv)))
        reach = max(reach, scale * (np.abs(q[h]) @ np.abs(kk).T).max())
    return out, err, lse, reach


def lse_bound(n, d, reach):
    """fp32 dot products of d terms, a sum of n exponentials, exp2 and log2 good to 2^-21."""
    return (d + 8) * 2.0 ** -24 * reach + n * 2.0 ** -24 + 2.0 ** -20


def sequence_bwd(q, k, v, do, window, sinks, scale):
    """One sequence: (dq, bound), (dk, bound), (dv, bound)."""
    G = q.shape[0] // k.shape[0]
    m = mask(q.shape[1], window, sinks)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    eq, ek, ev = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for h in range(q.shape[0]):
        kk, vv, qq, gg = k[h // G], v[h // G], q[h], do[h]
        p = attn.head_probs(qq, kk, m, scale)
        o = p @ vv
        oerr = U * np.abs(o) + 2 * U * (p @ np.abs(vv))
        dz = p * (gg @ vv.T - (gg * o).sum(1, keepdims=True))
        zerr = U * np.abs(dz) + p * (np.abs(gg) * oerr).sum(1, keepdims=True)
        dq[h] = scale * (dz @ kk)
        dk[h // G] += scale * (dz.T @ qq)
        dv[h // G] += p.T @ gg
        eq[h] = scale * (zerr @ np.abs(kk))
        ek[h // G] += scale * (zerr.T @ np.abs(qq))
        ev[h // G] += U * (p.T @ np.abs(gg))
    return tuple((x, ROOM * (e + U * np.abs(x))) for x, e in ((dq, eq), (dk, ek), (dv, ev)))
