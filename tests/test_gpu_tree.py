"""Drafted trees over the paged cache (tree_mask, cache_tree_attn) against the fp64 oracle: masks and positions equal,
outputs element by element within the bound of their roundings."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import tree as OT
from oracle import window as OW
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def _randn(seed, shape, gpu, mul=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * mul).to(BF).to(gpu)


def _dev(x, gpu):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).to(gpu)


def _parents(seed, B, T, kind="tree"):
    rng = np.random.default_rng(seed)
    t = np.arange(T)
    if kind == "chain":
        return np.tile(t - 1, (B, 1))
    if kind == "star":
        return np.full((B, T), -1)
    return (np.sqrt(rng.random((B, T))) * (t + 1)).astype(np.int64) - 1


def _filled(seed, contexts, T, Hkv, d, gpu, counts, kmul=1.0):
    """A pool of garbage (NaN codes too) with the tokens of every context and its nodes written."""
    g = torch.Generator().manual_seed(seed)
    total = [n + (T if counts is None else c) for n, c in zip(contexts, counts or [T] * len(contexts))]
    needs = [(n + 63) // 64 for n in total]
    pages = sum(needs) + 2
    cache = ms.make_cache(pages, Hkv, d, gpu)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).copy_(torch.randint(0, 256, t.shape, generator=g, dtype=torch.uint8))
    for t in (cache.k_scale, cache.v_scale):
        t.copy_(2.0 ** torch.randint(-9, 3, t.shape, generator=g).float())
    order = torch.randperm(pages, generator=g)
    table = torch.full((len(total), max(max(needs), 1)), -1, dtype=I32)
    at = 0
    for b, n in enumerate(needs):
        table[b, :n] = order[at:at + n].to(I32)
        at += n
    table = table.to(gpu)
    L = torch.tensor(total, dtype=I32, device=gpu)
    n = max(max(total), 1)
    k, v = _randn(seed + 1, (len(total), Hkv, n, d), gpu, kmul), _randn(seed + 2, (len(total), Hkv, n, d), gpu)
    ms.cache_append(cache, table, torch.zeros_like(L), k, v, counts=L)
    return cache, table, L


def _host(c):
    return [t.cpu().view(torch.uint8).numpy() for t in (c.k, c.v)] + \
           [t.cpu().numpy().astype(np.float64) for t in (c.k_scale, c.v_scale)]


def _check(q, out, lse, cache, table, L, sees, at, counts, W, S, scale=None):
    B, T, d = q.shape[0], q.shape[2], q.shape[3]
    lens = L.cpu().numpy()
    ro, eo, rl = OT.attention(to_f64(q.contiguous().cpu()), *_host(cache), table.cpu().numpy(), lens, sees, at,
                              counts or [T] * B, W, S, scale or d ** -0.5)
    go = to_f64(out.contiguous().cpu())
    assert np.isfinite(go).all()
    err = np.abs(go - ro)
    assert (err <= eo).all(), f"out off by {err.max():.3e}, {(err > eo).sum()} elements"
    gl = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(gl), np.isneginf(rl))
    fine = np.isfinite(rl)
    if fine.any():
        reach = 8.0 * max(1.0, float(q.double().abs().max())) * np.sqrt(d)
        assert np.abs(gl[fine] - rl[fine]).max() <= OW.lse_bound(int(lens.max()), d, reach)


def _masks(parents, contexts, counts, W, S):
    T = parents.shape[1]
    both = [OT.mask(parents[b], contexts[b], T if counts is None else counts[b], W, S) for b in range(len(contexts))]
    return np.stack([x[0] for x in both]), np.stack([x[1] for x in both])


def _run(gpu, Hq, Hkv, d, T, contexts, counts, W, S, kind="tree", seed=1, qmul=1.0, width=0):
    B = len(contexts)
    print(f"tree Hq{Hq} Hkv{Hkv} d{d} T{T} {contexts} {counts} W{W} S{S} {kind}", flush=True)
    parents = _parents(seed, B, T, kind)
    at, sees = _masks(parents, contexts, counts, W, S)
    cnt = None if counts is None else torch.tensor(counts, dtype=I32, device=gpu)
    gat, gseen = ms.tree_mask(_dev(parents, gpu), torch.tensor(contexts, dtype=I32, device=gpu), counts=cnt, window=W,
                              sinks=S)
    assert np.array_equal(gat.cpu().numpy(), at) and np.array_equal(gseen.cpu().numpy(), OT.words(sees))
    cache, table, L = _filled(T + d, contexts, T, Hkv, d, gpu, counts)
    narrow = table
    if width:
        table = torch.full((B, width), -1, dtype=I32, device=gpu)
        table[:, :narrow.shape[1]] = narrow
    q = _randn(seed, (B, Hq, T, d), gpu, qmul)
    out, lse = ms.cache_tree_attn(cache, table, L, q, gseen, positions=gat if W else None, counts=cnt, window=W, sinks=S)
    torch.cuda.synchronize()
    _check(q, out, lse, cache, narrow, L, sees, at, counts, W, S)
    again = ms.cache_tree_attn(cache, table, L, q, gseen, positions=gat, counts=cnt, window=W, sinks=S)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    return out, lse


@pytest.mark.parametrize("B,T,kind,W,S", [(1, 1, "tree", 0, 0), (3, 31, "tree", 0, 0), (2, 32, "chain", 5, 2),
                                          (2, 33, "star", 1, 0), (5, 64, "tree", 3, 100), (2, 257, "chain", 0, 0),
                                          (1, 1024, "tree", 4, 0), (300, 16, "tree", 0, 0)])
def test_masks_match_oracle(gpu, B, T, kind, W, S):
    rng = np.random.default_rng(T)
    contexts = [int(x) for x in rng.integers(0, 300, B)]
    counts = [int(x) for x in rng.integers(0, T + 1, B)]
    parents = _parents(T, B, T, kind)
    parents[0, -1] = T + 7   # no node before it: the context's child
    for cnt in (None, counts):
        at, sees = _masks(parents, contexts, cnt, W, S)
        gat, gseen = ms.tree_mask(_dev(parents, gpu), _dev(np.array(contexts), gpu), window=W, sinks=S,
                                  counts=None if cnt is None else _dev(np.array(cnt), gpu))
        assert np.array_equal(gat.cpu().numpy(), at) and np.array_equal(gseen.cpu().numpy(), OT.words(sees))


@pytest.mark.parametrize("Hq,Hkv,d,T,contexts,counts,W,S,kind", [
    (1, 1, 64, 1, [0], None, 0, 0, "tree"), (4, 1, 128, 1, [63, 64, 65], None, 0, 0, "tree"),
    (4, 2, 64, 8, [100, 0, 57], None, 0, 0, "tree"), (28, 4, 128, 16, [700, 50], None, 0, 0, "tree"),
    (28, 4, 128, 16, [130, 63, 0, 1], [16, 3, 0, 7], 0, 0, "tree"), (8, 8, 64, 33, [500], None, 0, 0, "tree"),
    (4, 1, 128, 64, [200, 64], [64, 1], 0, 0, "star"), (2, 1, 128, 100, [90], None, 0, 0, "chain"),
    (12, 4, 64, 61, [300, 1, 64], [61, 40, 0], 0, 0, "tree"), (16, 2, 64, 5, [300, 3], None, 40, 4, "tree"),
    (4, 2, 128, 70, [150, 20], [70, 33], 30, 2, "chain"), (8, 1, 64, 40, [333], None, 3, 0, "tree"),
    (4, 4, 128, 20, [257, 600], None, 100, 70, "tree"), (1, 1, 128, 300, [64, 10], [300, 150], 0, 0, "tree"),
    (3, 1, 64, 1024, [70], None, 0, 0, "tree"), (6, 2, 128, 7, [5, 9], None, 0, 300, "tree"),
])
def test_tree_attn_matches_oracle(gpu, Hq, Hkv, d, T, contexts, counts, W, S, kind):
    _run(gpu, Hq, Hkv, d, T, contexts, counts, W, S, kind)


@pytest.mark.parametrize("Hq,Hkv,d,T,contexts", [
    (4, 1, 64, 3, [20011, 1, 640, 0, 9000]), (28, 4, 128, 12, [8000, 100, 3001]), (8, 2, 128, 40, [5000, 2500]),
    (28, 4, 128, 8, [4000, 100, 3001]), (8, 2, 64, 16, [9000, 640, 0, 77]), (8, 1, 128, 300, [2000, 1]),
])
def test_tree_attn_long_and_ragged(gpu, Hq, Hkv, d, T, contexts):
    """Many chunks of one context beside short ones."""
    _run(gpu, Hq, Hkv, d, T, contexts, None, 0, 0, qmul=2.0)
    _run(gpu, Hq, Hkv, d, T, contexts, [max(1, T // (b + 1)) for b in range(len(contexts))], 1000, 100, qmul=2.0)


@pytest.mark.parametrize("B,Hq,Hkv,d,T", [(150, 2, 1, 64, 2), (60, 12, 4, 64, 6), (90, 8, 2, 128, 12), (40, 4, 4, 64, 40),
                                          (300, 2, 2, 128, 20)])
def test_tree_attn_many_sequences(gpu, B, Hq, Hkv, d, T):
    rng = np.random.default_rng(B)
    contexts = [int(x) for x in rng.integers(0, 300, B)]
    counts = [int(x) for x in rng.integers(0, T + 1, B)]
    _run(gpu, Hq, Hkv, d, T, contexts, counts, 0, 0)


@pytest.mark.parametrize("Hq,Hkv,d,T,contexts,width", [
    (4, 1, 64, 4, [1500, 700], 0), (4, 1, 64, 4, [600] * 130, 0), (4, 2, 128, 5, [5000, 90, 2500], 0),
    (16, 4, 128, 8, [3000, 90, 1500], 0), (8, 1, 64, 4, [4000, 1, 64], 0), (1, 1, 64, 12, [3, 1200], 150),
])
@pytest.mark.parametrize("W,S", [(0, 0), (900, 70)])
def test_few_rows_over_several_chunks(gpu, Hq, Hkv, d, T, contexts, width, W, S):
    rng = np.random.default_rng(T)
    _run(gpu, Hq, Hkv, d, T, contexts, [int(x) for x in rng.integers(1, T + 1, len(contexts))], W, S, width=width)


@pytest.mark.parametrize("d,Hq,T", [(64, 8, 64), (128, 4, 100)])
def test_many_tiles_of_rows(gpu, d, Hq, T):
    """From 512 tiles of 128 rows on, each walks its pages by itself, or, where the table is wide, one of several chunks."""
    rng = np.random.default_rng(T)
    contexts = [int(x) for x in rng.integers(0, 100, 128)]
    counts = [int(x) for x in rng.integers(0, T + 1, 128)]
    _run(gpu, Hq, 1, d, T, contexts, counts, 0, 0, width=7)
    contexts[77], contexts[90] = 4190, 4030
    _run(gpu, Hq, 1, d, T, contexts, counts, 0, 0, width=150)


def test_the_widest_table(gpu):
    """100 tiles in a table of 2^24 pages, which are dealt out by twos."""
    _run(gpu, 64, 1, 64, 200, [1500], None, 0, 0, width=2 ** 24)


def test_all_trees_empty(gpu):
    """No node anywhere; nodes of the last sequence alone."""
    for counts in ([0, 0, 0, 0], [0, 0, 0, 40], [40, 0, 0, 0]):
        _run(gpu, 8, 2, 64, 40, [300, 1000, 0, 700], counts, 0, 0)


@pytest.mark.parametrize("d", [64, 128])
def test_missing_pages_positions_and_strides_of_many_rows(gpu, d):
    Hq, Hkv, T, contexts = 12, 2, 50, [500, 130, 64]
    cache, table, L = _filled(8, contexts, T, Hkv, d, gpu, None)
    table[0, 1], table[0, 8], table[2, 1] = 10 ** 6, -1, -5
    q = _randn(1, (3, T, Hq, d), gpu).transpose(1, 2)
    at, sees = _masks(_parents(2, 3, T), contexts, None, 0, 0)
    seen = _dev(OT.words(sees), gpu)
    out = torch.empty((3, T, Hq, d), dtype=BF, device=gpu).transpose(1, 2)
    got, lse = ms.cache_tree_attn(cache, table, L, q, seen, scale=0.2, out=out)
    torch.cuda.synchronize()
    assert got is out
    _check(q, out, lse, cache, table, L, sees, at, None, 0, 0, 0.2)
    for odd in ([0, 50, 51], [-3, 7, 1]):
        n = torch.tensor(odd, dtype=I32, device=gpu)
        out, lse = ms.cache_tree_attn(cache, table, n, q, seen)
        torch.cuda.synchronize()
        _check(q, out, lse, cache, table, n.clamp(min=0), sees, at, None, 0, 0)
    far = torch.tensor([2 ** 31 - 1, 64 * table.shape[1] + 60, 2 ** 30], dtype=I32, device=gpu)
    out, lse = ms.cache_tree_attn(cache, table, far, q, seen, positions=far[:, None].expand(3, T).contiguous(), window=40)
    torch.cuda.synchronize()
    assert torch.isneginf(lse).all() and (out == 0).all()
    rng = np.random.default_rng(d)   # positions in any order, some outside the nodes' places
    at = np.stack([rng.integers(n - 30, n + T + 30, T) for n in contexts])
    at[:, :2] = 2 ** 31 - 1, -2 ** 31
    for W, S in ((1, 0), (50, 3), (70, 200)):
        out, lse = ms.cache_tree_attn(cache, table, L, q, seen, positions=_dev(at, gpu), window=W, sinks=S)
        torch.cuda.synchronize()
        _check(q, out, lse, cache, table, L, sees, at, None, W, S)


@pytest.mark.parametrize("d,T", [(64, 1), (128, 5), (64, 40), (128, 70)])
@pytest.mark.parametrize("W,S", [(0, 0), (30, 3)])
def test_chain_is_cache_attn(gpu, d, T, W, S):
    """A tree without branches sees what consecutive tokens see."""
    Hq, Hkv, contexts = 4, 2, [150, 64, 3]
    parents = _parents(0, 3, T, "chain")
    at, seen = ms.tree_mask(_dev(parents, gpu), _dev(np.array(contexts), gpu), window=W, sinks=S)
    cache, table, L = _filled(5, contexts, T, Hkv, d, gpu, None)
    q = _randn(1, (3, Hq, T, d), gpu)
    out, lse = ms.cache_tree_attn(cache, table, L, q, seen, positions=at, window=W, sinks=S)
    want, wl = ms.cache_attn(cache, table, L, q, window=W, sinks=S)
    at, sees = _masks(parents, contexts, None, W, S)
    _check(q, out, lse, cache, table, L, sees, at, None, W, S)
    _check(q, want, wl, cache, table, L, sees, at, None, W, S)


def test_any_masks_and_empty_rows(gpu):
    """Masks that are no tree's; rows without a key: out 0, lse -inf; bits behind the counts mean nothing."""
    Hq, Hkv, d, T, contexts, counts = 4, 2, 64, 40, [0, 70, 0], [40, 17, 5]
    rng = np.random.default_rng(0)
    sees = rng.random((3, T, T)) < 0.3
    sees[0, 3] = sees[0, 39] = False
    sees[2] = False
    cache, table, L = _filled(6, contexts, T, Hkv, d, gpu, counts)
    q, cnt = _randn(1, (3, Hq, T, d), gpu), torch.tensor(counts, dtype=I32, device=gpu)
    at = np.array(contexts)[:, None] + np.zeros((3, T), np.int64)
    for extra in (False, True):
        words = sees.copy()
        if extra:
            for b, c in enumerate(counts):
                words[b, :, c:] = True
                words[b, c:] = True
        out, lse = ms.cache_tree_attn(cache, table, L, q, _dev(OT.words(words), gpu), counts=cnt)
        torch.cuda.synchronize()
        _check(q, out, lse, cache, table, L, sees, at, counts, 0, 0)
        assert (out[0, :, [3, 39]] == 0).all() and torch.isneginf(lse[0, :, [3, 39]]).all()
        assert (out[2] == 0).all() and torch.isneginf(lse[2]).all() and (out[1, :, 17:] == 0).all()


def test_positions_outside_the_nodes_are_cut(gpu):
    Hq, Hkv, d, T, contexts, W, S = 2, 1, 64, 10, [200], 50, 3
    cache, table, L = _filled(7, contexts, T, Hkv, d, gpu, None)
    q = _randn(1, (1, Hq, T, d), gpu)
    _, sees = _masks(_parents(1, 1, T), contexts, None, W, S)
    at = np.array([[-7, 0, 199, 200, 205, 209, 210, 10 ** 9, -2 ** 31, 2 ** 31 - 1]])
    out, lse = ms.cache_tree_attn(cache, table, L, q, _dev(OT.words(sees), gpu), positions=_dev(at, gpu), window=W, sinks=S)
    torch.cuda.synchronize()
    _check(q, out, lse, cache, table, L, sees, at, None, W, S)


def test_missing_pages_lengths_and_garbage(gpu):
    """Tokens without a page are not seen; lengths below the counts, of zero, past the table; free slots and pages hold NaN."""
    Hq, Hkv, d, T, contexts = 4, 2, 64, 12, [300, 130, 64]
    cache, table, L = _filled(8, contexts, T, Hkv, d, gpu, None)
    table[0, 1], table[0, 3], table[2, 1] = 10 ** 6, -1, -5
    q = _randn(1, (3, Hq, T, d), gpu)
    at, sees = _masks(_parents(2, 3, T), contexts, None, 0, 0)
    seen = _dev(OT.words(sees), gpu)
    out, lse = ms.cache_tree_attn(cache, table, L, q, seen)
    torch.cuda.synchronize()
    _check(q, out, lse, cache, table, L, sees, at, None, 0, 0)
    for odd in ([0, 5, 12], [-3, 0, 1]):
        n = torch.tensor(odd, dtype=I32, device=gpu)
        out, lse = ms.cache_tree_attn(cache, table, n, q, seen)
        torch.cuda.synchronize()
        _check(q, out, lse, cache, table, n.clamp(min=0), sees, at, None, 0, 0)
    far = torch.tensor([2 ** 31 - 1, 64 * table.shape[1] + 20, 2 ** 30], dtype=I32, device=gpu)
    out, lse = ms.cache_tree_attn(cache, table, far, q, seen, positions=far[:, None].expand(3, T).contiguous(), window=40)
    torch.cuda.synchronize()
    assert torch.isneginf(lse).all() and (out == 0).all()


def test_nan_queries_stay_in_their_rows(gpu):
    Hq, Hkv, d, T, contexts = 8, 2, 128, 20, [400]
    cache, table, L = _filled(9, contexts, T, Hkv, d, gpu, None)
    q = _randn(1, (1, Hq, T, d), gpu)
    seen = ms.tree_mask(_dev(_parents(3, 1, T), gpu), L - T)[1]
    want, wl = ms.cache_tree_attn(cache, table, L, q, seen)
    q[0, 3, 7] = float("nan")
    out, lse = ms.cache_tree_attn(cache, table, L, q, seen)
    assert out[0, 3, 7].isnan().all() and lse[0, 3, 7].isnan()
    keep = torch.ones((Hq, T), dtype=torch.bool, device=gpu)
    keep[3, 7] = False
    assert torch.equal(out[0][keep], want[0][keep]) and torch.equal(lse[0][keep], wl[0][keep])


@pytest.mark.parametrize("d,T", [(64, 3), (128, 6), (64, 14), (128, 12), (64, 60), (128, 45)])
@pytest.mark.parametrize("W,S", [(100, 3), (65, 0), (200, 130)])
def test_nan_outside_the_window_and_behind_the_nodes(gpu, d, T, W, S):
    """Codes that no row sees may be NaN: those before every row's window and behind the sinks, nodes behind the counts."""
    Hq, Hkv, contexts, counts = 8, 2, [500, 300, 64], [T, max(T - 2, 1), T]
    cache, table, L = _filled(13, contexts, T, Hkv, d, gpu, None)
    q = _randn(1, (3, Hq, T, d), gpu)
    cnt = _dev(np.array(counts), gpu)
    total = _dev(np.array(contexts) + np.array(counts), gpu)
    at, seen = ms.tree_mask(_dev(_parents(5, 3, T), gpu), _dev(np.array(contexts), gpu), counts=cnt, window=W, sinks=S)
    want = ms.cache_tree_attn(cache, table, total, q, seen, positions=at, counts=cnt, window=W, sinks=S)
    assert want[0].isfinite().all()
    for b, n in enumerate(contexts):
        for j in list(range(S, n - W + 1)) + list(range(n + counts[b], n + T)):
            page = int(table[b, j // 64])
            cache.k.view(torch.uint8)[page, :, j % 64] = 0x7f
            cache.v.view(torch.uint8)[page, :, :, j % 64] = 0xff
    got = ms.cache_tree_attn(cache, table, total, q, seen, positions=at, counts=cnt, window=W, sinks=S)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("d,T", [(64, 4), (128, 8), (64, 14), (128, 60)])
def test_nan_keys_stay_with_the_rows_that_see_them(gpu, d, T):
    Hq, Hkv, contexts = 8, 2, [300, 62]
    at, sees = _masks(_parents(8, 2, T), contexts, None, 0, 0)
    cache, table, L = _filled(15, contexts, T, Hkv, d, gpu, None)
    q = _randn(3, (2, Hq, T, d), gpu)
    seen = _dev(OT.words(sees), gpu)
    want = ms.cache_tree_attn(cache, table, L, q, seen)
    node = T // 2
    for b, n in enumerate(contexts):
        cache.k.view(torch.uint8)[int(table[b, (n + node) // 64]), :, (n + node) % 64, 3] = 0x7f
    out, lse = ms.cache_tree_attn(cache, table, L, q, seen)
    hit = torch.from_numpy(sees[:, :, node]).to(gpu)[:, None].expand(2, Hq, T)
    assert hit.any() and not hit.all()
    assert out[hit].isnan().all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], want[0][~hit]) and torch.equal(lse[~hit], want[1][~hit])


def _unseen(sees, at, contexts, counts, W, S):
    """Of each sequence: which of its slots no node sees."""
    out = []
    for b, (n, m) in enumerate(zip(contexts, counts)):
        j = np.arange(n)
        p = np.clip(at[b, :m], n, n + m - 1)[:, None]
        context = (p - j < W) | (j < S) if W else np.ones((m, n), bool)
        out.append(~np.concatenate([context.any(0), sees[b, :m, :m].any(0)]) if m else np.ones(n, bool))
    return out


@pytest.mark.parametrize("Hq,Hkv,d,T,contexts,counts,W,S,late", [
    (2, 2, 64, 1, [65], None, 1, 0, False), (8, 2, 64, 4, [500, 90, 62], [4, 3, 2], 0, 0, False),
    (8, 2, 128, 3, [63, 300], None, 0, 0, False), (4, 2, 64, 16, [500, 64], None, 30, 3, True),
    (2, 2, 128, 30, [500, 200], None, 77, 0, True), (4, 4, 64, 30, [500, 564], [30, 29], 77, 5, True),
    (8, 2, 64, 14, [200, 513, 40], [14, 12, 1], 0, 0, False), (8, 2, 128, 14, [500, 120], None, 70, 0, True),
    (8, 2, 64, 45, [130, 500], None, 60, 2, True), (8, 2, 128, 45, [130, 500], [45, 40], 0, 0, False),
    (2, 2, 64, 200, [70, 500], [200, 190], 0, 0, False), (2, 2, 128, 200, [640, 30], None, 100, 70, True),
    (1, 1, 64, 1024, [30], None, 0, 0, False), (16, 2, 128, 130, [300], None, 140, 0, True),
    (4, 1, 64, 4, [1500, 700], None, 600, 70, True), (8, 2, 128, 40, [5000, 700], None, 0, 0, False),
    (8, 1, 64, 64, [20] * 77 + [4500] + [33] * 52, None, 0, 0, False),
    (8, 1, 128, 64, [4200] + [70] * 129, None, 4100, 0, True),
])
def test_tokens_that_no_node_sees_may_hold_anything(gpu, Hq, Hkv, d, T, contexts, counts, W, S, late):
    """Pruned nodes, and the context between what the window reaches from the first place and from the first position given:
    codes NaN, and scales that are no numbers of pages where that is all."""
    print(f"unseen Hq{Hq} Hkv{Hkv} d{d} T{T} {contexts} {counts} W{W} S{S}", flush=True)
    B, live = len(contexts), counts or [T] * len(contexts)
    rng = np.random.default_rng(T + d)
    at, sees = _masks(_parents(6, B, T), contexts, counts, W, S)
    gone = rng.random((B, T)) < 0.4
    gone[:, T // 3:T // 3 + 130] = T > 64   # whole pages of them
    gone[:, 0] = True
    sees &= ~gone[:, None, :]
    if late:
        at = np.array(contexts)[:, None] + np.array(live)[:, None] - 1 - rng.integers(0, 2, (B, T))
    cache, table, L = _filled(14, contexts, T, Hkv, d, gpu, counts)
    q = _randn(2, (B, Hq, T, d), gpu)
    cnt = None if counts is None else _dev(np.array(counts), gpu)
    args = dict(positions=_dev(at, gpu), counts=cnt, window=W, sinks=S)
    want = ms.cache_tree_attn(cache, table, L, q, _dev(OT.words(sees), gpu), **args)
    torch.cuda.synchronize()
    _check(q, *want, cache, table, L, sees, at, counts, W, S)
    odd = [float("nan"), float("inf"), -float("inf"), -1.0]
    planted = 0
    for b, none in enumerate(_unseen(sees, at, contexts, live, W, S)):
        slots = np.flatnonzero(none)
        planted += len(slots)
        pages = _dev(table[b].cpu().numpy()[slots // 64], gpu).long()
        where = _dev(slots % 64, gpu).long()
        cache.k.view(torch.uint8)[pages, :, where] = 0x7f
        cache.v.view(torch.uint8)[pages, :, :, where] = 0xff
        for lp in range((len(none) + 63) // 64):
            if none[64 * lp:64 * lp + 64].all():
                cache.k_scale[int(table[b, lp])] = odd[lp % 4]
                cache.v_scale[int(table[b, lp])] = odd[(lp + 1) % 4]
    assert planted
    got = ms.cache_tree_attn(cache, table, L, q, _dev(OT.words(sees), gpu), **args)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [24, 7, 70])
def test_magnitudes_of_queries_and_scales(gpu, T, d):
    """Queries of one large and many small columns, tiny and huge ones, and page scales that are no powers of two and far
    apart."""
    Hq, Hkv, contexts = 4, 2, [500]
    cache, table, L = _filled(10, contexts, T, Hkv, d, gpu, None)
    g = torch.Generator().manual_seed(3)
    cache.k_scale.copy_(cache.k_scale.cpu() * (1 + torch.rand(cache.k_scale.shape, generator=g)))
    cache.v_scale.copy_(cache.v_scale.cpu() * (1 + torch.rand(cache.v_scale.shape, generator=g)) *
                        2.0 ** torch.randint(-20, 20, cache.v_scale.shape, generator=g).float())
    q = _randn(1, (1, Hq, T, d), gpu)
    q[0, 0] *= 2.0 ** -100
    q[0, 1, :, 5] *= 2.0 ** 7
    q[0, 1, :, 9:] *= 2.0 ** -12
    q[0, 2] *= 0
    q[0, 3] *= 16
    at, sees = _masks(_parents(4, 1, T), contexts, None, 0, 0)
    out, lse = ms.cache_tree_attn(cache, table, L, q, _dev(OT.words(sees), gpu))
    torch.cuda.synchronize()
    _check(q, out, lse, cache, table, L, sees, at, None, 0, 0)


def test_strides_scale_and_outputs(gpu):
    Hq, Hkv, d, T, contexts = 6, 2, 64, 9, [100, 333]
    cache, table, L = _filled(11, contexts, T, Hkv, d, gpu, None)
    q = _randn(1, (2, T, Hq, d), gpu).transpose(1, 2)
    seen = ms.tree_mask(_dev(_parents(5, 2, T), gpu), L - T)[1]
    out = torch.empty((2, T, Hq, d), dtype=BF, device=gpu).transpose(1, 2)
    got, lse = ms.cache_tree_attn(cache, table, L, q, seen, scale=0.3, out=out)
    want, wl = ms.cache_tree_attn(cache, table, L, q.contiguous(), seen, scale=0.3)
    assert got is out and torch.equal(got, want) and torch.equal(lse, wl)
    at, sees = _masks(_parents(5, 2, T), contexts, None, 0, 0)
    _check(q, out, lse, cache, table, L, sees, at, None, 0, 0, 0.3)


def test_two_graphs_and_a_stream(gpu):
    """Two captured calls of other sizes with workspaces of their own, replayed in turn on changing inputs; a call on a side
    stream."""
    made = []
    for T, d, ctx in ((12, 64, [900, 20]), (40, 128, [3000, 700])):
        cache, table, L = _filled(12 + T, ctx, T, 2, d, gpu, None)
        q = _randn(T, (2, 4, T, d), gpu)
        seen = ms.tree_mask(_dev(_parents(T, 2, T), gpu), L - T)[1]
        ms.cache_tree_attn(cache, table, L, q, seen)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = ms.cache_tree_attn(cache, table, L, q, seen)
        made.append((graph, got, cache, table, L, q, seen))
    for seed in range(3):
        for graph, got, cache, table, L, q, seen in made:
            q.copy_(_randn(seed, q.shape, gpu))
        for graph, *_ in made:
            graph.replay()
        for graph, got, cache, table, L, q, seen in made:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            want = ms.cache_tree_attn(cache, table, L, q, seen, stream=side)
            torch.cuda.current_stream().wait_stream(side)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
