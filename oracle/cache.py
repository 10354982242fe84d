"""Reference paged 8-bit cache: append with rotation, attention over the pages.

Test infrastructure; see oracle/__init__.py.  All arithmetic is fp64, one token
and one page at a time.  Codes are e4m3 (1 sign, 4 exponent bits of bias 7, 3
mantissa bits; 0x7f and 0xff NaN, no infinities) with a power-of-two scale per
page and head: the smallest s >= 2^-126 with |x| <= 448 s.
"""
import numpy as np

from . import attn

PAGE = 64


def _decode_table():
    t = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        t[c] = np.nan if c & 127 == 127 else (-x if c & 128 else x)
    return t


DECODE = _decode_table()
_MAGNITUDES = DECODE[:127]


def encode(x):
    """Codes of the nearest e4m3 values, ties to the even code; what is not finite: NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.abs(x)
    fine = np.isfinite(x)
    a = np.where(fine, a, 0.0)
    hi = np.clip(np.searchsorted(_MAGNITUDES, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up = _MAGNITUDES[hi] - a
    down = a - _MAGNITUDES[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(np.signbit(x), code | 128, code)
    return np.where(fine, code, 127).astype(np.uint8)


def scale_of(amax):
    if not amax > 0:
        return 2.0 ** -126
    m, e = np.frexp(amax)
    return max(2.0 ** (int(e) - (9 if m <= 0.875 else 8)), 2.0 ** -126)


def rotate(x, pos, freq):
    """x [T, d] at the positions pos: columns (i, i + d/2) turn by pos freq[i]."""
    if freq is None:
        return x.copy()
    h = x.shape[1] // 2
    a = pos[:, None].astype(np.float64) * np.asarray(freq, np.float64)[None]
    c, s = np.cos(a), np.sin(a)
    return np.concatenate([x[:, :h] * c - x[:, h:] * s, x[:, h:] * c + x[:, :h] * s], 1)


def append(k, v, ks, vs, table, lens, knew, vnew, counts, freq):
    """k [P, H, 64, d], v [P, H, d, 64] uint8 codes and ks, vs [P, H]: updated in place."""
    for b in range(len(lens)):
        t = 0
        while t < counts[b]:
            pos = int(lens[b]) + t
            lp, o = pos // PAGE, pos % PAGE
            m = min(PAGE - o, int(counts[b]) - t)
            if lp < table.shape[1] and 0 <= table[b, lp] < k.shape[0]:
                page = table[b, lp]
                for h in range(k.shape[1]):
                    x = rotate(knew[b, h, t:t + m], np.arange(pos, pos + m), freq)
                    for new, codes, scale in ((x, k[page, h], ks), (vnew[b, h, t:t + m], v[page, h].T, vs)):
                        fine = np.abs(new[np.isfinite(new)])
                        need = scale_of(fine.max() if fine.size else 0.0)
                        was = float(scale[page, h])
                        now = max(need, was) if o else need
                        if o and now > was:
                            with np.errstate(invalid="ignore"):
                                codes[:o] = encode(DECODE[codes[:o]] * (was / now))
                        with np.errstate(invalid="ignore"):
                            codes[o:o + m] = encode(new / now)
                        scale[page, h] = now
            t += m


def gather(k, v, ks, vs, table, n, b, hk):
    """Keys, values [n, d] of sequence b and which of its tokens have a page."""
    pos = np.arange(n)
    lp = pos // PAGE
    page = np.where(lp < table.shape[1], table[b, np.minimum(lp, table.shape[1] - 1)], -1)
    have = (page >= 0) & (page < k.shape[0])
    page = np.where(have, page, 0)
    kk = DECODE[k[page, hk, pos % PAGE]] * ks[page, hk][:, None]
    vv = DECODE[v[page, hk, :, pos % PAGE]] * vs[page, hk][:, None]
    return kk, vv, have


def attention(q, k, v, ks, vs, table, lens, window, sinks, scale):
    """q [B, Hq, T, d] -> out, its bound (see oracle/window.py), lse."""
    B, Hq, T, d = q.shape
    G = Hq // k.shape[1]
    out, err, lse = np.zeros_like(q), np.zeros_like(q), np.full((B, Hq, T), -np.inf)
    for b in range(B):
        n = int(lens[b])
        i = n - T + np.arange(T)[:, None]
        j = np.arange(n)[None]
        for h in range(Hq):
            if n == 0:
                continue
            kk, vv, have = gather(k, v, ks, vs, table, n, b, h // G)
            m = (j <= i) & ((i - j < (window or n + 1)) | (j < sinks)) & have[None]
            seen = attn.seen_keys(m)
            if seen.size == 0:
                continue
            kk, vv, m = kk[seen], vv[seen], m[:, seen]
            out[b, h], lse[b, h] = attn.head_fwd(q[b, h], kk, vv, m, scale)
            p = attn.head_probs(q[b, h], kk, m, scale)
            err[b, h] = (1 + 2.0 ** -4) * (2.0 ** -8 * np.abs(out[b, h]) + 2.0 ** -8 * (p @ np.abs(vv)))
    return out, err, lse
