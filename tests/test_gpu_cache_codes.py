"""Every code that cache_append leaves in the pool, one by one: a new key's code is that of the fp64 rotated value moved
by no more than the fp32 rotation may (2^-22 of |x1| + |x2|: cos and sin rounded, a product and a sum rounded, 2^-24
each), a new value's and a moved older token's code is exact, and all other codes and scales are those from before."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import cache as OC
from tests.helpers import to_f64
from tests.test_gpu_cache import _freq, _host, _pool, _randn, _same, _table


def _expected(before, table, lens, k, v, counts, freq):
    """(lowest, nearest, highest) K codes, V codes, scales after the append of k, v [B, H, T, d] to `before`."""
    kc, vc, ks, vs = [x.copy() for x in before]
    lo, hi = kc.copy(), kc.copy()
    B, H, _, d = k.shape
    for b in range(B):
        for lp in range(int(lens[b]) // OC.PAGE, (int(lens[b]) + counts[b] + OC.PAGE - 1) // OC.PAGE):
            p0, p1 = max(lens[b], OC.PAGE * lp), min(lens[b] + counts[b], OC.PAGE * (lp + 1))
            if p1 <= p0 or lp >= table.shape[1] or not 0 <= table[b, lp] < kc.shape[0]:
                continue
            page, o, e = table[b, lp], p0 - OC.PAGE * lp, p1 - OC.PAGE * lp
            for h in range(H):
                new, x = k[b, h, p0 - lens[b]:p1 - lens[b]], v[b, h, p0 - lens[b]:p1 - lens[b]]
                rot = OC.rotate(new, np.arange(p0, p1), freq)
                off = np.abs(new[:, :d // 2]) + np.abs(new[:, d // 2:])
                off = 2.0 ** -22 * np.concatenate([off, off], 1) * (freq is not None)
                for y, scale, codes in ((rot, ks, (kc, lo, hi)), (x, vs, (vc,))):
                    was, need = scale[page, h], OC.scale_of(np.abs(y).max())
                    now = max(was, need) if o else need
                    scale[page, h] = now
                    for i, c in enumerate(codes):
                        c = c[page, h] if scale is ks else c[page, h].T
                        if o and now > was:
                            with np.errstate(invalid="ignore"):
                                c[:o] = OC.encode(OC.DECODE[c[:o]] * (was / now))
                        c[o:e] = OC.encode((y + (0, -off, off)[i]) / now)
    return lo, kc, hi, vc, ks, vs


def _check_codes(got, want):
    lo, mid, hi, vc, ks, vs = want
    k, v, gs, gv = got
    assert np.array_equal(gs, ks) and np.array_equal(gv, vs), "scales"
    fits = _same(k, lo) | _same(k, mid) | _same(k, hi)
    assert fits.all(), f"{(~fits).sum()} K codes, first at {np.argwhere(~fits)[0]}"
    fits = _same(v, vc)
    assert fits.all(), f"{(~fits).sum()} V codes, first at {np.argwhere(~fits)[0]}"


def _append(gpu, cache, table, lens, T, counts, d, freq, seed, kmul=1.0):
    B, H = len(lens), cache.k.shape[1]
    k, v = (_randn(seed + i, (B, H, T, d), gpu, kmul) for i in range(2))
    before = _host(cache)
    dev = lambda x: torch.from_numpy(np.asarray(x, np.int32)).to(gpu)  # noqa: E731
    ms.cache_append(cache, dev(table), dev(lens), k, v, inv_freq=freq, counts=dev(counts))
    torch.cuda.synchronize()
    want = _expected(before, table, lens, to_f64(k.cpu()), to_f64(v.cpu()), counts, None if freq is None else freq.cpu().numpy())
    _check_codes(_host(cache), want)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,d,T,counts", [
    ([0], 1, 64, 1, [1]), ([64, 1, 1000], 2, 64, 1, [1, 1, 1]), ([63, 62], 4, 128, 2, [2, 2]),
    ([0, 63], 4, 64, 65, [65, 65]), ([5, 64, 127], 2, 128, 130, [130, 0, 77]), ([60, 0, 12, 200], 2, 64, 7, [7, 1, 0, 5]),
    ([37], 8, 128, 700, [700]), ([131000], 1, 128, 90, [90]),
])
def test_append_codes(gpu, lens, H, d, T, counts):
    print(f"codes {lens} H{H} d{d} T{T} {counts}", flush=True)
    needs = [(n + T + 63) // 64 for n in lens]
    cache, table = _pool(T + d, sum(needs) + 2, H, d, gpu), _table(T, needs, sum(needs) + 2)
    _append(gpu, cache, table, [0] * len(lens), max(max(lens), 1), lens, d, None, 100)
    _append(gpu, cache, table, lens, T, counts, d, _freq(d, gpu), 200)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_append_codes_of_growing_tokens(gpu, d):
    """One token after the other, each raising its page's scale: old codes move, and exactly so."""
    cache, table = _pool(3, 4, 2, d, gpu), _table(1, [2], 4)
    for t in range(70):
        _append(gpu, cache, table, [t], 1, [1], d, _freq(d, gpu), 300 + t, kmul=2.0 ** (t % 12 - 6))


def test_code_check_sees_one_wrong_code():
    """Truncation instead of rounding, a neighbour's code, a touched slot: each is seen (planted in the expected codes)."""
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((1, 1, 9, 16)), rng.standard_normal((1, 1, 9, 16))
    pool = [rng.integers(0, 127, s, dtype=np.uint8) for s in ((2, 1, 64, 16), (2, 1, 16, 64))] + [np.ones((2, 1)) / 64] * 2
    freq = 100.0 ** -np.arange(8)
    want = _expected(pool, np.array([[1]]), [3], k, v, [9], freq)
    lo, mid, hi, vc, ks, vs = want
    _check_codes((mid, vc, ks, vs), want)
    moved = np.argwhere((lo == hi) & (mid & 127 > 1) & (mid & 127 < 126))
    for at in (tuple(moved[0]), tuple(moved[-1]), (0, 0, 5, 3), (1, 0, 40, 0)):
        for codes, i in ((mid, 0), (vc, 1)):
            bad = codes.copy()
            x = at if i == 0 else (at[0], at[1], at[3], at[2])
            bad[x] ^= 1
            with pytest.raises(AssertionError):
                _check_codes((bad, vc, ks, vs) if i == 0 else (mid, bad, ks, vs), want)
