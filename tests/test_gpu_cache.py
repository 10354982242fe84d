"""The paged 8-bit cache (cache_append, cache_attn) against the fp64 oracle.

Append: scales equal the oracle's and codes too, except where the value lies so
near the middle of two codes that fp32 rotation decides (see _codes_match).
Attention: element by element within the bound of its roundings to bf16."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import cache as OC
from oracle import window as OW
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _randn(seed, shape, gpu, mul=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * mul).to(BF).to(gpu)


def _freq(d, gpu, base=10000.0):
    return (base ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).float().to(gpu)


def _pool(seed, pages, Hkv, d, gpu):
    """A cache of random codes (NaN among them) and scales: a pool that other sequences used."""
    g = torch.Generator().manual_seed(seed)
    c = ms.make_cache(pages, Hkv, d, gpu)
    for t in (c.k, c.v):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8))
    for t in (c.k_scale, c.v_scale):
        t.copy_(2.0 ** torch.randint(-9, 3, t.shape, generator=g).float())
    return c


def _host(c):
    return [t.cpu().view(torch.uint8).numpy().copy() for t in (c.k, c.v)] + \
           [t.cpu().numpy().astype(np.float64) for t in (c.k_scale, c.v_scale)]


def _table(seed, needs, pages, width=None):
    order = np.random.default_rng(seed).permutation(pages)
    t = np.full((len(needs), width or max(max(needs), 1)), -1, np.int32)
    at = 0
    for b, n in enumerate(needs):
        t[b, :n] = order[at:at + n]
        at += n
    return t


def _same(got, want):
    """Equal codes; 0x7f and 0xff are both NaN, and the sign of a NaN stands for nothing."""
    return (got == want) | ((got & 127 == 127) & (want & 127 == 127))


def _codes_match(name, got, want):
    """Equal codes, or neighbours: fp32 products and sums move a rotated value by at most 2^-22 of |x1| + |x2|, so a
    code may differ where the value lies that near the middle of two; fewer than one value in a thousand does."""
    same = _same(got, want)
    g, w = OC.DECODE[got[~same]], OC.DECODE[want[~same]]
    assert np.isfinite(g).all() and np.isfinite(w).all(), name
    assert (np.abs(g - w) <= np.maximum(2.0 ** -9, 0.134 * np.maximum(np.abs(g), np.abs(w)))).all(), name
    assert (~same).mean() <= 1e-3, f"{name}: {(~same).mean():.2e} of the codes differ"


def _append_and_check(gpu, cache, table, lens, T, counts, Hq, d, freq, seed, kmul=1.0, strided=False):
    B, Hkv = len(lens), cache.k.shape[1]
    shape = lambda h: (B, T, h, d) if strided else (B, h, T, d)  # noqa: E731
    q, k, v = (_randn(seed + i, shape(h), gpu, m) for i, (h, m) in enumerate(((Hq, 1.0), (Hkv, kmul), (Hkv, kmul))))
    if strided:
        q, k, v = (t.transpose(1, 2) for t in (q, k, v))
    ref = _host(cache)
    dev = lambda x: torch.from_numpy(np.asarray(x, np.int32)).to(gpu)  # noqa: E731
    q_out = torch.full((B, Hq, T, d), 7.0, dtype=BF, device=gpu)
    ms.cache_append(cache, dev(table), dev(lens), k, v, q=q, inv_freq=freq, q_out=q_out,
                    counts=None if counts is None else dev(counts))
    torch.cuda.synchronize()
    n = [T] * B if counts is None else counts
    fr = None if freq is None else freq.cpu().numpy()
    f = [to_f64(t.contiguous().cpu()) for t in (q, k, v)]
    OC.append(*ref, table, lens, f[1], f[2], n, fr)
    got = _host(cache)
    assert np.array_equal(got[2], ref[2]) and np.array_equal(got[3], ref[3]), "scales"
    _codes_match("k", got[0], ref[0])
    assert _same(got[1], ref[1]).all(), "v codes"
    qo = to_f64(q_out.cpu())
    for b in range(B):   # rows past the counts too
        for h in range(Hq):
            r = OC.rotate(f[0][b, h], int(lens[b]) + np.arange(T), fr)
            err = np.abs(qo[b, h] - r)
            assert (err <= 2.0 ** -8 * np.abs(r) + 2.0 ** -20).all()
    return q_out


@pytest.mark.parametrize("B,Hq,Hkv,d,T,lens,counts", [
    (1, 1, 1, 64, 1, [0], None), (1, 4, 1, 128, 1, [63], None), (3, 4, 2, 64, 1, [64, 1, 1000], None),
    (2, 7, 1, 128, 2, [63, 62], None), (2, 4, 4, 64, 65, [0, 63], None), (1, 2, 2, 128, 200, [37], None),
    (3, 4, 2, 128, 130, [5, 64, 127], [130, 0, 77]), (4, 8, 2, 64, 7, [60, 0, 12, 200], [7, 1, 0, 5]),
    (2, 28, 4, 128, 64, [64, 128], None),
])
def test_append_matches_oracle(gpu, B, Hq, Hkv, d, T, lens, counts):
    print(f"append B{B} Hq{Hq} Hkv{Hkv} d{d} T{T} {lens} {counts}", flush=True)
    needs = [(n + T + 63) // 64 for n in lens]
    pages = sum(needs) + 2
    cache = _pool(T + d, pages, Hkv, d, gpu)
    table = _table(T, needs, pages)
    # the tokens already there are written by an append, without rotation
    if max(lens):
        _append_and_check(gpu, cache, table, [0] * B, max(lens), lens, Hq, d, None, 100)
    _append_and_check(gpu, cache, table, lens, T, counts, Hq, d, _freq(d, gpu), 200, strided=T > 1)


def test_append_moves_older_tokens_to_a_larger_scale(gpu):
    """One token after the other, each about twice as large: every one raises its page's scale."""
    Hkv, d = 2, 64
    cache = _pool(3, 4, Hkv, d, gpu)
    table = _table(1, [2], 4)
    for t in range(70):
        _append_and_check(gpu, cache, table, [t], 1, None, 2, d, _freq(d, gpu), 300 + t, kmul=2.0 ** (t % 12 - 6))


def test_append_scale_borders(gpu):
    """Largest values at and around 448 s, zeros alone, tiny and huge values, infinities and NaN."""
    d = 64
    tops = [448.0, 450.0, 446.0, 0.0, 1.0, 2.0 ** -130, 3e38, 7.0, 2.0 ** -120]
    k = torch.zeros((len(tops), 1, 3, d), dtype=BF)
    for b, top in enumerate(tops):
        k[b, 0, 0] = torch.linspace(-top, top, d, dtype=torch.float64).to(BF)
    k[4, 0, 1, 5], k[4, 0, 1, 6], k[4, 0, 2, 7] = float("inf"), float("-inf"), float("nan")
    k = k.to(gpu)
    B = len(tops)
    cache = _pool(8, B, 1, d, gpu)
    table = torch.arange(B, dtype=torch.int32, device=gpu).view(B, 1)
    ref = _host(cache)
    ms.cache_append(cache, table, torch.zeros(B, dtype=torch.int32, device=gpu), k, k)
    torch.cuda.synchronize()
    f = to_f64(k.cpu())
    OC.append(*ref, table.cpu().numpy(), [0] * B, f, f, [3] * B, None)
    got = _host(cache)
    assert np.array_equal(got[2], ref[2]) and np.array_equal(got[3], ref[3])
    for a, b in zip(got[:2], ref[:2]):
        nan = np.isnan(OC.DECODE[b])
        assert np.array_equal(np.isnan(OC.DECODE[a]), nan) and np.array_equal(a[~nan], b[~nan])


@pytest.mark.parametrize("pos", [0, 1, 999, 131071, 1048575, 100000007, 2 ** 30 - 64])
def test_append_rotation_of_far_positions(gpu, pos):
    """Angles of far positions are reduced in 64 bits: the rotated queries to bf16's rounding.  (No page is held
    there, so only the queries are written.)"""
    d = 128
    cache = _pool(5, 1, 1, d, gpu)
    before = _host(cache)
    table = torch.full((1, 1), -1, dtype=torch.int32, device=gpu)
    q, k = _randn(1, (1, 3, 4, d), gpu), _randn(2, (1, 1, 4, d), gpu)
    freq = _freq(d, gpu, 500000.0)
    got = ms.cache_append(cache, table, torch.tensor([pos], dtype=torch.int32, device=gpu), k, k, q=q, inv_freq=freq)
    torch.cuda.synchronize()
    for h in range(3):
        r = OC.rotate(to_f64(q[0, h].cpu()), pos + np.arange(4), freq.cpu().numpy())
        assert (np.abs(to_f64(got[0, h].cpu()) - r) <= 2.0 ** -8 * np.abs(r) + 2.0 ** -20).all()
    for a, b in zip(_host(cache), before):
        assert np.array_equal(a, b, equal_nan=True)


def test_append_without_a_page_is_dropped(gpu):
    """Entries outside the pool and tokens past the table write nothing; the tokens with a page are written."""
    d, B = 64, 3
    cache = _pool(6, 3, 2, d, gpu)
    table = np.array([[0, 99], [-1, 1], [2, -5]], np.int32)
    _append_and_check(gpu, cache, table, [10, 10, 100], 130, None, 2, d, _freq(d, gpu), 400)


def test_append_in_place(gpu):
    d = 64
    q, k = _randn(1, (2, 4, 5, d), gpu), _randn(2, (2, 2, 5, d), gpu)
    cache = _pool(9, 4, 2, d, gpu)
    table = torch.arange(4, dtype=torch.int32, device=gpu).view(2, 2)
    lens = torch.tensor([3, 62], dtype=torch.int32, device=gpu)
    want = ms.cache_append(cache, table, lens, k, k, q=q, inv_freq=_freq(d, gpu))
    assert ms.cache_append(cache, table, lens, k, k, q=q, inv_freq=_freq(d, gpu), q_out=q) is q
    assert torch.equal(q, want)


# ---------------------------------------------------------------- attention
def _filled(seed, lens, Hkv, d, gpu, extra=2, kmul=1.0):
    """A pool of garbage with the tokens of every sequence written into their pages."""
    needs = [(n + 63) // 64 for n in lens]
    pages = sum(needs) + extra
    cache = _pool(seed, pages, Hkv, d, gpu)
    table = torch.from_numpy(_table(seed, needs, pages)).to(gpu)
    n = max(max(lens), 1)
    k, v = _randn(seed + 1, (len(lens), Hkv, n, d), gpu, kmul), _randn(seed + 2, (len(lens), Hkv, n, d), gpu)
    zero = torch.zeros(len(lens), dtype=torch.int32, device=gpu)
    L = torch.tensor(lens, dtype=torch.int32, device=gpu)
    ms.cache_append(cache, table, zero, k, v, inv_freq=_freq(d, gpu), counts=L)
    return cache, table, L


def _attn_check(q, out, lse, cache, table, lens, W, S, scale=None):
    ref = _host(cache)
    d = q.shape[3]
    ro, eo, rl = OC.attention(to_f64(q.contiguous().cpu()), *ref, table.cpu().numpy(), lens, W, S, scale or d ** -0.5)
    err = np.abs(to_f64(out.contiguous().cpu()) - ro)
    assert np.isfinite(err).all()
    assert (err <= eo).all(), f"out off by {err.max():.3e}"
    gl = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(gl), np.isneginf(rl))
    fine = np.isfinite(rl)
    if fine.any():
        reach = 8.0 * max(1.0, float(q.double().abs().max())) * np.sqrt(d)   # scale sum |q||k|, generously
        bound = OW.lse_bound(max(lens), d, reach)
        assert np.abs(gl[fine] - rl[fine]).max() <= bound


@pytest.mark.parametrize("Hq,Hkv,d,T,lens,W,S", [
    (1, 1, 64, 1, [1], 0, 0), (4, 1, 128, 1, [64, 65, 63], 0, 0), (28, 4, 128, 1, [700, 3, 0, 129], 0, 0),
    (8, 8, 64, 1, [1000, 257], 0, 0), (4, 2, 64, 1, [900, 70], 100, 4), (4, 1, 128, 1, [2000], 64, 130),
    (16, 1, 64, 1, [500], 0, 0), (17, 1, 64, 1, [500, 20], 0, 0), (8, 1, 128, 4, [300, 2, 66], 0, 0),
    (4, 2, 128, 5, [400, 64], 33, 1), (7, 1, 64, 9, [777], 0, 0), (4, 1, 128, 40, [300, 40, 39, 1], 0, 0),
    (2, 2, 64, 200, [450, 200], 70, 5), (16, 2, 128, 33, [130, 900], 128, 64), (4, 1, 64, 65, [65], 0, 0),
    (3, 1, 64, 1, [640], 1, 0), (3, 1, 64, 2, [640], 1, 1),
])
def test_attn_matches_oracle(gpu, Hq, Hkv, d, T, lens, W, S):
    print(f"attn Hq{Hq} Hkv{Hkv} d{d} T{T} {lens} W{W} S{S}", flush=True)
    cache, table, L = _filled(T + d, lens, Hkv, d, gpu)
    q = _randn(1, (len(lens), Hq, T, d), gpu)
    out, lse = ms.cache_attn(cache, table, L, q, window=W, sinks=S)
    torch.cuda.synchronize()
    _attn_check(q, out, lse, cache, table, lens, W, S)


def test_attn_long_and_ragged(gpu):
    """Many chunks of one sequence beside short ones; repeated calls give the same bits."""
    lens = [20011, 1, 640, 0, 9000]
    cache, table, L = _filled(11, lens, 1, 64, gpu)
    q = _randn(1, (5, 4, 1, 64), gpu, 2.0)
    out, lse = ms.cache_attn(cache, table, L, q)
    again = ms.cache_attn(cache, table, L, q)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    _attn_check(q, out, lse, cache, table, lens, 0, 0)


def test_attn_bad_pages_and_lengths(gpu):
    """Tokens without a page are not seen; a sequence without any is empty; lengths past the table end with it."""
    lens = [300, 200, 130]
    cache, table, L = _filled(12, lens, 2, 64, gpu)
    table[0, 1] = 10 ** 6
    table[0, 3] = -1
    table[1] = -1
    q = _randn(1, (3, 4, 3, 64), gpu)
    out, lse = ms.cache_attn(cache, table, L, q)
    torch.cuda.synchronize()
    _attn_check(q, out, lse, cache, table, lens, 0, 0)
    assert (out[1] == 0).all() and torch.isneginf(lse[1]).all()
    longer = torch.tensor([64 * table.shape[1] + 5, 2 ** 31 - 1, -7], dtype=torch.int32, device=gpu)
    out, lse = ms.cache_attn(cache, table, longer, q)
    torch.cuda.synchronize()
    assert torch.isneginf(lse[2]).all() and (out[2] == 0).all()


def test_attn_free_slots_hold_anything(gpu):
    """Codes of free slots and of tokens outside the window do not reach the result, NaN included."""
    lens = [150, 70, 321]
    cache, table, L = _filled(13, lens, 2, 128, gpu)
    q = _randn(1, (3, 4, 1, 128), gpu)
    for W, S in ((0, 0), (40, 3)):
        want = ms.cache_attn(cache, table, L, q, window=W, sinks=S)
        soiled = ms.Cache(*(t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)))
        k, v = soiled.k.view(torch.uint8), soiled.v.view(torch.uint8)
        for b, n in enumerate(lens):
            for p in range((n + 63) // 64):
                for s in range(64):
                    pos = 64 * p + s
                    if pos >= n or (W and pos <= n - 1 - W and pos >= S):
                        k[table[b, p], :, s] = 0x7f
                        v[table[b, p], :, :, s] = 0xff
        got = ms.cache_attn(soiled, table, L, q, window=W, sinks=S)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_attn_strides_and_scale(gpu):
    lens = [100, 333]
    cache, table, L = _filled(14, lens, 2, 64, gpu)
    q = _randn(1, (2, 6, 4, 64), gpu).transpose(1, 2)   # [B, T, Hq, d] memory
    out = torch.empty((2, 6, 4, 64), dtype=BF, device=gpu).transpose(1, 2)
    got, lse = ms.cache_attn(cache, table, L, q, scale=0.3, out=out)
    want, wl = ms.cache_attn(cache, table, L, q.contiguous(), scale=0.3)
    assert torch.equal(got, want) and torch.equal(lse, wl)
    _attn_check(q, out, lse, cache, table, lens, 0, 0, 0.3)


def test_decode_loop_together(gpu):
    """A prefill into the cache, then tokens one by one (append, lens, attention) in a captured graph, against the
    training operator on the same tokens: the cache's 8-bit rounding apart, the same attention."""
    B, Hq, Hkv, d, W, S, n0, steps = 2, 4, 2, 64, 48, 4, 100, 40
    n = n0 + steps
    q, k, v = (_randn(i, (B, h, n, d), gpu) for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    cache = _pool(15, 2 * 3 + 1, Hkv, d, gpu)
    table = torch.arange(6, dtype=torch.int32, device=gpu).view(2, 3)
    freq = _freq(d, gpu)
    lens = torch.zeros(B, dtype=torch.int32, device=gpu)
    pre = ms.cache_append(cache, table, lens, k[:, :, :n0], v[:, :, :n0], q=q[:, :, :n0], inv_freq=freq)
    lens += n0
    outs = [ms.cache_attn(cache, table, lens, pre, window=W, sinks=S)[0]]
    sq, sk, sv = (t[:, :, :1].clone() for t in (q, k, v))

    def step():
        r = ms.cache_append(cache, table, lens, sk, sv, q=sq, inv_freq=freq)
        lens.add_(1)
        return ms.cache_attn(cache, table, lens, r, window=W, sinks=S)[0]

    keep = [t.clone() for t in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale, lens)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t, old in zip((cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale, lens), keep):
        t.copy_(old)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for t in range(n0, n):
        for a, b in ((sq, q), (sk, k), (sv, v)):
            a.copy_(b[:, :, t:t + 1])
        graph.replay()
        outs.append(got.clone())
        _ = (got.float() + 1).sum().item()   # eager work and a wait between the replays
    assert lens.tolist() == [n, n]
    out = torch.cat(outs, 2)
    # the codes that a token had when a row saw it may have moved to a larger scale since; so compare with the
    # attention over the unquantised tokens, whose K and V differ from the codes by at most 2^-4 (twice rounded: 2^-3)
    rot = lambda x: torch.from_numpy(np.stack([np.stack([OC.rotate(h, np.arange(n), freq.cpu().numpy()) for h in b])  # noqa: E731
                                               for b in to_f64(x.cpu())]))
    win = ms.make_window(B, n, Hq, Hkv, d, W, S)
    want, _ = ms.window_fwd(win, rot(q).to(BF).to(gpu), rot(k).to(BF).to(gpu), v)
    err = (out.double() - want.double()).abs()
    assert float(err.max()) < 0.5 and float((err.square().sum() / want.double().square().sum()).sqrt()) < 0.1


# ---------------------------------------------------------------- many sequences, long tables
def _some_lens(seed, B, top):
    lens = np.random.default_rng(seed).integers(0, top + 1, B)
    lens[::9] = 0
    lens[1] = top
    return [int(x) for x in lens]


@pytest.mark.parametrize("B,Hq,Hkv,d,T,top,wide", [
    (150, 2, 1, 64, 1, 700, 0),      # equal chunks over more than 64 tiles
    (100, 4, 2, 128, 1, 600, 0),     # a workgroup per tile
    (3, 4, 2, 64, 1, 2000, 0), (40, 12, 4, 64, 1, 3000, 0), (200, 16, 1, 64, 1, 1500, 0),   # one of many waves
    (800, 1, 1, 64, 1, 300, 150),    # chunks from the table's width, most tables half empty
    (30, 12, 4, 128, 2, 400, 130), (4200, 1, 1, 64, 1, 150, 0), (2, 20, 1, 128, 1, 9000, 0),
    (40, 4, 4, 64, 40, 500, 0), (70, 8, 2, 128, 70, 300, 140),
])
def test_attn_many_sequences(gpu, B, Hq, Hkv, d, T, top, wide):
    print(f"attn B{B} Hq{Hq} Hkv{Hkv} d{d} T{T} top{top} width{wide}", flush=True)
    lens = _some_lens(B, B, top)
    cache, table, L = _filled(B, lens, Hkv, d, gpu)
    if wide > table.shape[1]:
        more = torch.full((B, wide), -1, dtype=torch.int32, device=gpu)
        more[:, :table.shape[1]] = table
        table = more
    q = _randn(1, (B, Hq, T, d), gpu)
    out, lse = ms.cache_attn(cache, table, L, q)
    again = ms.cache_attn(cache, table, L, q)
    torch.cuda.synchronize()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    _attn_check(q, out, lse, cache, table, lens, 0, 0)


def test_attn_one_long_among_many_short(gpu):
    """Chunks of a fixed length: one context of many, the others of one."""
    B, Hkv = 800, 1
    lens = [20] * B
    lens[5], lens[799] = 30000, 12345
    cache, table, L = _filled(21, [20] * B, Hkv, 64, gpu, extra=700)
    wide = torch.full((B, 470), -1, dtype=torch.int32, device=gpu)
    wide[:, :1] = table
    free = torch.tensor(sorted(set(range(cache.k.shape[0])) - set(table[:, 0].tolist())), dtype=torch.int32)
    assert len(free) >= 469 + 192
    wide[5, 1:469], wide[799, 1:193] = free[:468].to(gpu), free[468:660].to(gpu)
    for i, b in enumerate((5, 799)):
        n = lens[b] - 20
        part = torch.tensor([20], dtype=torch.int32, device=gpu)
        k, v = _randn(30 + i, (1, Hkv, n, 64), gpu), _randn(40 + i, (1, Hkv, n, 64), gpu)
        ms.cache_append(cache, wide[b:b + 1].contiguous(), part, k, v, inv_freq=_freq(64, gpu))
    L = torch.tensor(lens, dtype=torch.int32, device=gpu)
    q = _randn(1, (B, 4, 1, 64), gpu, 2.0)
    for W, S in ((0, 0), (9000, 100)):
        out, lse = ms.cache_attn(cache, wide, L, q, window=W, sinks=S)
        torch.cuda.synchronize()
        _attn_check(q, out, lse, cache, wide, lens, W, S)


@pytest.mark.parametrize("Hq,Hkv,d,T,L", [(4, 1, 64, 600, 1500), (2, 1, 128, 1100, 1700)])
def test_attn_many_rows_in_chunks(gpu, Hq, Hkv, d, T, L):
    """Row tiles whose chunks are joined a row per group of lanes."""
    cache, table, lens = _filled(T, [L], Hkv, d, gpu)
    q = _randn(1, (1, Hq, T, d), gpu)
    out, lse = ms.cache_attn(cache, table, lens, q)
    torch.cuda.synchronize()
    _attn_check(q, out, lse, cache, table, [L], 0, 0)


@pytest.mark.parametrize("B,Hq,Hkv,d,T,ragged", [(300, 3, 1, 64, 3, True), (1, 2, 1, 128, 36000, False),
                                                 (260, 2, 2, 128, 1, False)])
def test_append_of_many_pages(gpu, B, Hq, Hkv, d, T, ragged):
    """Several heads in a workgroup, and many pages."""
    rng = np.random.default_rng(T)
    lens = [int(x) for x in rng.integers(0, 130, B)]
    counts = [int(x) for x in rng.integers(0, T + 1, B)] if ragged else None
    needs = [(n + T + 63) // 64 for n in lens]
    cache = _pool(T, sum(needs) + 2, Hkv, d, gpu)
    table = _table(T, needs, sum(needs) + 2)
    _append_and_check(gpu, cache, table, [0] * B, max(lens), lens, Hq, d, None, 500)
    _append_and_check(gpu, cache, table, lens, T, counts, Hq, d, _freq(d, gpu), 600)


def test_attn_missing_page_beside_a_soiled_scale(gpu):
    """A token without a page is not seen, whatever the scales of the pool's first page hold."""
    for T, lens in ((1, [300, 90]), (1, [40 * 64, 200]), (40, [300, 90])):
        cache, table, L = _filled(17, lens, 2, 64, gpu, extra=3)
        held = set(table.flatten().tolist())
        if 0 in held:   # page 0 to be nobody's
            spare = next(p for p in range(1, cache.k.shape[0]) if p not in held)
            for t in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale):
                t[spare] = t[0]
            table[table == 0] = spare
        table[0, 2] = -1
        q = _randn(1, (2, 4, T, 64), gpu)
        want = ms.cache_attn(cache, table, L, q)
        for bad in (float("nan"), float("inf")):
            cache.k_scale[0] = cache.v_scale[0] = bad
            got = ms.cache_attn(cache, table, L, q)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        cache.k_scale[0] = cache.v_scale[0] = 1.0
        _attn_check(q, got[0], got[1], cache, table, lens, 0, 0)


def test_cache_beyond_4_gb(gpu):
    """Pages whose codes lie past 2^32 bytes: the same codes and results as in a small pool."""
    B, Hq, Hkv, d, pages = 2, 8, 8, 128, 70000
    big, small = ms.make_cache(pages, Hkv, d, gpu), ms.make_cache(8, Hkv, d, gpu)
    near = torch.arange(6, dtype=torch.int32, device=gpu).view(B, 3)
    far = near + (pages - 6)
    freq, lens = _freq(d, gpu), torch.tensor([0, 0], dtype=torch.int32, device=gpu)
    q, k, v = (_randn(i, (B, h, 150, d), gpu) for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    got = []
    for c, table in ((big, far), (small, near)):
        r = ms.cache_append(c, table, lens, k, v, q=q, inv_freq=freq)
        got.append((r,) + ms.cache_attn(c, table, lens + 150, r) + ms.cache_attn(c, table, lens + 150, r[:, :, :1]))
    for a, b in zip(*got):
        assert torch.equal(a, b)
    for p in range(6):
        m = 22 if p % 3 == 2 else 64   # the third page of a sequence holds 22 tokens, and anything behind them
        assert torch.equal(big.k[pages - 6 + p, :, :m].view(torch.uint8), small.k[p, :, :m].view(torch.uint8))
        assert torch.equal(big.v[pages - 6 + p, :, :, :m].view(torch.uint8), small.v[p, :, :, :m].view(torch.uint8))


def test_cache_two_calls_at_once(gpu):
    """Two streams read one cache, each with its own workspace and results."""
    lens = [9000, 300, 77]
    cache, table, L = _filled(23, lens, 2, 128, gpu)
    qs = [_randn(i, (3, 8, 1, 128), gpu) for i in (1, 2)]
    want = [ms.cache_attn(cache, table, L, q) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(5):
        got = [ms.cache_attn(cache, table, L, q, stream=s) for q, s in zip(qs, streams)]
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("B,Hq,Hkv,d,T,top,wide,W,S", [
    (800, 1, 1, 64, 1, 700, 150, 200, 3), (10, 4, 2, 64, 1, 4000, 0, 300, 0), (10, 4, 2, 128, 1, 4000, 0, 1000, 70),
    (220, 2, 1, 128, 1, 3000, 140, 700, 130), (9, 12, 4, 128, 3, 5000, 0, 64, 0), (20, 8, 1, 64, 60, 2500, 0, 500, 4),
    (150, 8, 2, 128, 70, 1500, 200, 300, 0),
])
def test_attn_many_sequences_in_a_window(gpu, B, Hq, Hkv, d, T, top, wide, W, S):
    """The window bounds the pages that are walked, and with them the split; the workspace is that of any window."""
    lens = _some_lens(B, B, top)
    cache, table, L = _filled(B, lens, Hkv, d, gpu)
    if wide > table.shape[1]:
        more = torch.full((B, wide), -1, dtype=torch.int32, device=gpu)
        more[:, :table.shape[1]] = table
        table = more
    q = _randn(1, (B, Hq, T, d), gpu)
    room = torch.empty(ms.cache_attn_workspace_bytes(cache, table, Hq, T), dtype=torch.uint8, device=gpu)
    out, lse = ms.cache_attn(cache, table, L, q, window=W, sinks=S, workspace=room)
    torch.cuda.synchronize()
    _attn_check(q, out, lse, cache, table, lens, W, S)
