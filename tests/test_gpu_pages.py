"""Moves in the paged cache (cache_keep, cache_fork) against the oracle, exact; and a loop of speculative decoding."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import cache as OC
from oracle import pages as OP
from oracle import tree as OT
from oracle import window as OW
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu
I32, BF = torch.int32, torch.bfloat16


def _pool(seed, pages, Hkv, d, gpu, nan=True):
    """A pool of random codes (NaN among them) and scales."""
    g = torch.Generator().manual_seed(seed)
    c = ms.make_cache(pages, Hkv, d, gpu)
    for t in (c.k, c.v):
        t.view(torch.uint8).copy_(torch.randint(0, 256 if nan else 0x7f, t.shape, generator=g, dtype=torch.uint8))
    for t in (c.k_scale, c.v_scale):
        t.copy_(2.0 ** torch.randint(-6, 4, t.shape, generator=g).float())
    return c


def _host(c):
    return [t.cpu().view(torch.uint8).numpy().copy() for t in (c.k, c.v)] + \
           [t.cpu().numpy().astype(np.float64) for t in (c.k_scale, c.v_scale)]


def _dev(x, gpu):
    return torch.from_numpy(np.ascontiguousarray(x).astype(np.int32)).to(gpu)


def _same(got, want):
    return (got == want) | ((got & 127 == 127) & (want & 127 == 127))


def _equal(cache, ref):
    got = _host(cache)
    assert np.array_equal(got[2], ref[2]) and np.array_equal(got[3], ref[3]), "scales"
    assert _same(got[0], ref[0]).all(), f"k: {(~_same(got[0], ref[0])).sum()} codes"
    assert _same(got[1], ref[1]).all(), f"v: {(~_same(got[1], ref[1])).sum()} codes"


def _table(seed, needs, pages, width=None):
    order = np.random.default_rng(seed).permutation(pages)
    t = np.full((len(needs), width or max(max(needs), 1)), -1, np.int32)
    at = 0
    for b, n in enumerate(needs):
        t[b, :n] = order[at:at + n]
        at += n
    return t


# ---------------------------------------------------------------- keep
def _keep(gpu, Hkv, d, T, lens, counts, path, kept, table=None, seed=0, cache=None):
    B = len(lens)
    print(f"keep Hkv{Hkv} d{d} T{T} {lens} {counts} {kept}", flush=True)
    needs = [(max(n, 0) + 63) // 64 for n in lens]
    cache = cache or _pool(seed, sum(needs) + 3, Hkv, d, gpu)
    table = _table(seed, needs, sum(needs) + 3) if table is None else table
    ref = _host(cache)
    ms.cache_keep(cache, _dev(table, gpu), _dev(np.array(lens), gpu), _dev(path, gpu), _dev(np.array(kept), gpu),
                  counts=None if counts is None else _dev(np.array(counts), gpu))
    torch.cuda.synchronize()
    OP.keep(*ref, table, np.maximum(lens, 0), path, kept, counts or [T] * B)
    _equal(cache, ref)
    return cache


def _paths(seed, B, T, counts, share):
    rng = np.random.default_rng(seed)
    path, kept = np.zeros((B, T), np.int64), []
    for b in range(B):
        take = np.flatnonzero(rng.random(T if counts is None else counts[b]) < share)
        path[b, :len(take)] = take
        kept.append(len(take))
    return path, kept


@pytest.mark.parametrize("Hkv,d,T,lens,counts,share", [
    (1, 64, 1, [1], None, 1.0), (1, 64, 2, [2, 65, 64], None, 0.5), (2, 128, 16, [70, 16, 128, 129, 140], None, 0.3),
    (4, 64, 40, [100, 64, 41], [40, 7, 0], 0.5), (8, 128, 16, [1000, 66], None, 0.2), (1, 128, 200, [263, 200, 500], None, 0.3),
    (3, 64, 130, [130, 300], [130, 129], 0.9), (2, 64, 300, [1024], None, 0.05), (1, 64, 64, [128, 127], None, 1.0),
])
def test_keep_matches_oracle(gpu, Hkv, d, T, lens, counts, share):
    for seed in range(3):
        path, kept = _paths(seed, len(lens), T, counts, share)
        _keep(gpu, Hkv, d, T, lens, counts, path, kept, seed=seed)


def test_keep_moves_tokens_between_scales(gpu):
    """Large tokens into a page of a small scale and the other way round: the page's older tokens follow, exactly or
    rounded below the normal range."""
    Hkv, d, T = 2, 64, 70
    for up in (-8, -3, 0, 3, 8, 14):
        cache = _pool(1, 4, Hkv, d, gpu, nan=False)
        table = np.array([[2, 0, 3]], np.int32)
        cache.k_scale.fill_(2.0 ** -3)
        cache.v_scale.fill_(2.0 ** -3)
        for t in (cache.k_scale, cache.v_scale):
            t[0] *= 2.0 ** up
            t[3] *= 2.0 ** (up / 2)   # no power of two for odd `up`
        path = np.zeros((1, T), np.int64)
        path[0, :6] = [3, 30, 31, 40, 66, 69]
        _keep(gpu, Hkv, d, T, [130], None, path, [6], table=table, cache=cache)


def test_keep_odd_paths_and_missing_pages(gpu):
    """Entries that do not ascend past their place, beyond the counts or without a page leave their place; kept beyond the
    counts is cut; lengths below the counts."""
    path = np.zeros((4, 20), np.int64)
    path[0, :6] = [0, 0, 5, 3, 19, 25]
    path[1, :3] = [-4, 2 ** 31 - 1, 7]
    path[2] = np.arange(20) + 1
    path[3, :4] = [1, 2, 4, 5]
    table = np.array([[0, 1], [2, 3], [4, -1], [5, 99]], np.int32)
    cache = _pool(3, 6, 2, 128, gpu)
    # (the same path once more: of rows 0, 3 the sources of 3, 3 -> places 3, 4)
    path[0, 3] = 3
    _keep(gpu, 2, 128, 20, [80, 75, 70, 6], None, path, [6, 3, 100, 4], table=table, cache=cache)
    _keep(gpu, 2, 128, 20, [80, 0, -5, 1], [20, 20, 20, 20], path, [0, 5, 5, -3], table=table, cache=cache)


def test_keep_in_a_graph_and_on_a_stream(gpu):
    Hkv, d, T, lens = 2, 64, 16, [70, 200]
    needs = [(n + 63) // 64 for n in lens]
    caches = [_pool(5, sum(needs), Hkv, d, gpu) for _ in range(3)]
    table = _dev(_table(5, needs, sum(needs)), gpu)
    L, path, kept = _dev(np.array(lens), gpu), _dev(np.zeros((2, T)), gpu), _dev(np.zeros(2), gpu)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ms.cache_keep(caches[0], table, L, path, kept)
    for seed in range(3):
        p, n = _paths(seed, 2, T, None, 0.4)
        path.copy_(_dev(p, gpu))
        kept.copy_(_dev(np.array(n), gpu))
        graph.replay()
        ms.cache_keep(caches[1], table, L, path, kept)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ms.cache_keep(caches[2], table, L, path, kept, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        a, b, c = (_host(x) for x in caches)
        for x, y, z in zip(a, b, c):
            assert np.array_equal(x, y, equal_nan=True) and np.array_equal(x, z, equal_nan=True)


# ---------------------------------------------------------------- fork
def _fork(gpu, cache, table, lens, refs, src, room, in_place=False):
    pages = cache.k.shape[0]
    ref = _host(cache)
    want = OP.fork(table, lens, refs, src, room, pages)
    dev_refs = _dev(refs, gpu)
    got = ms.cache_fork(cache, _dev(table, gpu), _dev(np.array(lens), gpu), dev_refs, _dev(np.array(src), gpu),
                        room=None if room is None else _dev(np.array(room), gpu), refs_out=dev_refs if in_place else None)
    torch.cuda.synchronize()
    got = [t.cpu().numpy() for t in got]
    for name, g, w in zip(("table", "lens", "refs", "missing"), got, want):
        assert np.array_equal(g, w), (name, g, w)
    for of, to in want[4]:
        for t in ref:
            t[to] = t[of]
    _equal(cache, ref)
    # the counts are those of the entries
    held = np.array(refs, np.int64)
    for t, sign in ((table, -1), (got[0], 1)):
        np.add.at(held, t[(t >= 0) & (t < pages)], sign)
    assert np.array_equal(held, got[2])
    return got


def _some(seed, B, N, width, pages, top, spare=0):
    rng = np.random.default_rng(seed)
    lens = [int(x) for x in rng.integers(0, min(top, 64 * width) + 1, B)]
    held = [min(width, (n + 63) // 64 + int(rng.integers(0, spare + 1))) for n in lens]
    table = _table(seed, held, pages, width)
    refs = np.zeros(pages, np.int64)
    np.add.at(refs, table[table >= 0], 1)
    refs[rng.integers(0, pages, 3)] += 1   # other tables' pages
    src = [int(x) for x in rng.integers(-1, B, N)]
    return table, lens, refs, src, rng


@pytest.mark.parametrize("B,N,width,pages,Hkv,d,top,spare", [
    (1, 1, 1, 4, 1, 64, 64, 0), (1, 3, 4, 20, 2, 64, 200, 1), (4, 4, 5, 40, 2, 128, 300, 1), (3, 9, 6, 70, 1, 64, 380, 2),
    (8, 2, 4, 60, 2, 64, 250, 0), (20, 60, 9, 800, 1, 64, 500, 1), (5, 300, 3, 1500, 1, 64, 190, 1), (2, 5, 300, 2000, 1, 64, 19000, 3),
    (300, 40, 2, 900, 1, 64, 128, 1), (2, 2, 5, 40000, 1, 64, 300, 1),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_fork_matches_oracle(gpu, B, N, width, pages, Hkv, d, top, spare, in_place):
    print(f"fork B{B} N{N} width{width} pages{pages} Hkv{Hkv} d{d}", flush=True)
    table, lens, refs, src, rng = _some(B + N, B, N, width, pages, top, spare)
    cache = _pool(B, pages, Hkv, d, gpu)
    room = [int(x) for x in rng.integers(-3, 64 * width + 50, N)]
    _fork(gpu, cache, table, lens, refs, src, None, in_place)
    _fork(gpu, cache, table, lens, refs, src, room, in_place)


@pytest.mark.parametrize("B,N,width,pages,top,spare", [
    (3, 5, 40, 25000, 2500, 2), (30, 40, 1300, 9000, 14000, 4), (2, 1100, 4, 3000, 250, 1), (200, 300, 12, 21000, 700, 1),
    (1, 1024, 2, 2100, 128, 1), (40, 33, 800, 12000, 15000, 9), (8, 256, 1024, 14000, 15000, 9), (1000, 256, 8, 9000, 450, 1), (1400, 256, 6, 11000, 350, 1),
    (4000, 200, 2, 9000, 100, 0), (8, 256, 1024, 9000, 15000, 9), (8, 257, 1024, 9000, 15000, 9),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_fork_of_large_pools_and_tables(gpu, B, N, width, pages, top, spare, in_place):
    """Either side of what one workgroup's memory holds."""
    print(f"fork B{B} N{N} width{width} pages{pages}", flush=True)
    table, lens, refs, src, rng = _some(B * N, B, N, width, pages, top, spare)
    cache = _pool(B, pages, 1, 64, gpu)
    room = [int(x) for x in rng.integers(-3, 64 * width + 50, N)]
    for want in (None, room):
        _fork(gpu, cache, table, lens, refs, src, want, in_place)


def test_fork_asks_for_2e31_pages(gpu):
    """More places than 32 bits count: the first rows get what there is, the others nothing."""
    pages, width, N = 50, 32800, 65536
    cache = _pool(1, pages, 1, 64, gpu)
    table = torch.full((1, width), -1, dtype=I32, device=gpu)
    zero = torch.zeros(1, dtype=I32, device=gpu)
    room = torch.full((N,), 64 * width, dtype=I32, device=gpu)
    got, lens, refs, missing = ms.cache_fork(cache, table, zero, torch.zeros(pages, dtype=I32, device=gpu),
                                             torch.full((N,), -1, dtype=I32, device=gpu), room=room)
    assert got[0, :pages].tolist() == list(range(pages)) and (got[0, pages:] == -1).all()
    assert all((part == -1).all() for part in got[1:].split(4096))
    assert (refs == 1).all() and (lens == 0).all()
    assert missing[0] == width - pages and (missing[1:] == width).all()


def test_fork_rows_that_ask_for_2e24_pages_each(gpu):
    """128 rows of the widest table ask for 2^31 pages, more than 32 bits count in one pass over the rows: the first row gets
    what there is, the others nothing."""
    pages, width, N = 50, 2 ** 24, 131
    print(f"fork N{N} width{width}", flush=True)
    cache = _pool(1, pages, 1, 64, gpu)
    table = torch.full((1, width), -1, dtype=I32, device=gpu)
    table[0, :2] = torch.tensor([7, 3], dtype=I32)
    refs = torch.zeros(pages, dtype=I32, device=gpu)
    refs[[3, 7]] = 1
    lens = torch.tensor([128], dtype=I32, device=gpu)
    src = torch.full((N,), -1, dtype=I32, device=gpu)
    src[-1] = 0
    room = torch.full((N,), 64 * width, dtype=I32, device=gpu)
    got, lens, refs, missing = ms.cache_fork(cache, table, lens, refs, src, room=room)
    free = [p for p in range(pages) if p not in (3, 7)]
    assert got[0, :pages - 2].tolist() == free and all((part == -1).all() for part in got[0, pages - 2:].split(1 << 22))
    assert all((row == -1).all() for row in got[1:-1])
    assert got[-1, :2].tolist() == [7, 3] and (got[-1, 2:] == -1).all()
    assert (refs == 1).all() and lens.tolist() == [0] * (N - 1) + [128]
    assert missing.tolist() == [width - pages + 2] + [width] * (N - 2) + [width - 2]


def test_fork_runs_out_of_pages(gpu):
    """Fewer free pages than are asked for: the first rows get theirs, the others' entries stay -1, a row whose last page
    could not be copied ends with its full pages."""
    table = np.array([[0, 1, -1, -1], [2, -1, -1, -1]], np.int32)
    refs = np.array([1, 1, 1, 0, 0, 1], np.int64)
    cache = _pool(1, 6, 2, 64, gpu)
    for src, room in (([0, 0, 0, 0, 0], None), ([0, 1, 0, 0, 1], [256] * 5), ([1, 1, 1], [64, 70, 256]), ([-1, 0], [300, 0])):
        got = _fork(gpu, cache, table, [100, 30], refs, src, room)
        if src == [0, 0, 0, 0, 0]:   # page 2 is given back: three copies' places, and four are asked for
            assert got[1].tolist() == [100, 100, 100, 100, 64] and got[3].tolist() == [0, 0, 0, 0, 1]


def test_fork_of_a_partly_filled_page_that_another_table_holds(gpu):
    """The first that continues the sequence shares it as before; the second one's copy is its own, and an append to that
    leaves the held page as it was."""
    Hkv, d = 2, 64
    cache = _pool(4, 6, Hkv, d, gpu, nan=False)
    got = _fork(gpu, cache, np.array([[4, 2, -1]], np.int32), [100], np.array([0, 0, 2, 0, 2, 0]), [0, 0], [100, 110])
    assert got[0].tolist() == [[4, 2, -1], [4, 0, -1]] and got[2].tolist() == [1, 0, 2, 0, 3, 0]
    before = _host(cache)
    g = torch.Generator().manual_seed(0)
    k = (torch.randn((1, Hkv, 10, d), generator=g) * 1000).to(BF).to(gpu)
    ms.cache_append(cache, _dev(got[0][1:], gpu), _dev(np.array([100]), gpu), k, k)
    after = _host(cache)
    for x, y in zip(before, after):
        assert not np.array_equal(x[0], y[0]) and np.array_equal(x[1:], y[1:])


def test_fork_frees_and_reuses(gpu):
    """Sequences that nothing continues give their pages back, and the same call allots them again; all freed at the end;
    entries and lengths out of range."""
    table = np.array([[0, 1, 2], [3, 4, -1], [5, 77, -2]], np.int32)
    refs = np.array([1, 1, 1, 1, 1, 1], np.int64)
    cache = _pool(2, 6, 1, 128, gpu)
    _fork(gpu, cache, table, [150, 128, 190], refs, [1, 1, -1, 1], [190, 140, 60, 128])
    _fork(gpu, cache, table, [10 ** 9, -5, 64], refs, [0, 1, 2, 7, -2 ** 31], [0, 64, 130, 5, 5])
    got = _fork(gpu, cache, table, [150, 128, 190], refs, [-1], None)
    assert (got[2] == 0).all() and (got[0] == -1).all()


def test_fork_in_a_graph(gpu):
    B, N, width, pages = 4, 12, 6, 90
    cache = _pool(3, pages, 2, 64, gpu)
    table, lens, refs, src, _ = _some(3, B, N, width, pages, 300)
    dt, dl, dr, ds = _dev(table, gpu), _dev(np.array(lens), gpu), _dev(refs, gpu), _dev(np.array(src), gpu)
    room = torch.full((N,), 350, dtype=I32, device=gpu)
    ms.cache_fork(cache, dt, dl, dr, ds, room=room)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ms.cache_fork(cache, dt, dl, dr, ds, room=room)
    for seed in range(4, 8):
        table, lens, refs, src, _ = _some(seed, B, N, width, pages, 300)
        for t, x in ((dt, table), (dl, lens), (dr, refs), (ds, src)):
            t.copy_(_dev(np.array(x), gpu))
        graph.replay()
        _ = (got[0].float() + 1).sum().item()
        want = OP.fork(table, lens, refs, src, [350] * N, pages)
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("d,axes", [(64, 1), (128, 3)])
def test_speculative_decoding_together(gpu, d, axes):
    """Prompts into pages that fork allots; rounds of drafting: room, tree_mask, append at its positions, tree attention,
    the accepted path kept; forks between the rounds; all freed at the end.  After every round the attention of the last
    accepted token, appended again on its own, equals that of a cache built token by token from the accepted ones, up to the
    codes that moved to another scale; tables and counts stay those of their entries."""
    B, Hq, Hkv, T, pages, width, W, S = 3, 4, 2, 12, 60, 8, 90, 4
    rng = np.random.default_rng(d)
    g = torch.Generator().manual_seed(d)
    rand = lambda *s: torch.randn(s, generator=g).to(BF).to(gpu)  # noqa: E731
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).float().to(gpu)
    axis = (torch.arange(d // 2) % axes).to(I32).to(gpu)
    many = lambda at: (at[None] * torch.arange(1, axes + 1, dtype=I32, device=gpu)[:, None, None]).contiguous()  # noqa: E731
    cache = _pool(9, pages, Hkv, d, gpu)
    table = torch.full((B, width), -1, dtype=I32, device=gpu)
    lens, refs = torch.zeros(B, dtype=I32, device=gpu), torch.zeros(pages, dtype=I32, device=gpu)
    prompt = [50, 64, 117]
    table, lens, refs, missing = ms.cache_fork(cache, table, lens, refs, torch.arange(B, dtype=I32, device=gpu),
                                               room=_dev(np.array(prompt), gpu))
    assert not missing.any() and lens.tolist() == [0] * B
    k, v = rand(B, Hkv, 117, d), rand(B, Hkv, 117, d)
    at = torch.arange(117, dtype=I32, device=gpu).expand(B, 117)
    counts = _dev(np.array(prompt), gpu)
    ms.cache_append(cache, table, lens, k, v, inv_freq=freq, counts=counts, positions=many(at), axis=axis)
    lens = lens + counts
    told = [[(k[b, :, t], v[b, :, t]) for t in range(prompt[b])] for b in range(B)]   # the tokens so far
    for step in range(4):
        if step in (1, 3):   # beams change: one twice, one given up
            src = [2, 0, 2] if step == 1 else [0, 0, 1]
            table, lens, refs, missing = ms.cache_fork(cache, table, lens, refs, _dev(np.array(src), gpu),
                                                       room=(lens[src] + T).to(I32))
            told = [list(told[s]) for s in src]
        else:
            table, lens, refs, missing = ms.cache_fork(cache, table, lens, refs, torch.arange(B, dtype=I32, device=gpu),
                                                       room=lens + T)
        assert not missing.any()
        held = np.zeros(pages, np.int64)
        entries = table.cpu().numpy()
        np.add.at(held, entries[entries >= 0], 1)
        assert np.array_equal(held, refs.cpu().numpy())
        parents = ((np.sqrt(rng.random((B, T))) * (np.arange(T) + 1)).astype(np.int64) - 1)
        nodes = rng.integers(1, T + 1, B)
        q, k, v = rand(B, Hq, T, d), rand(B, Hkv, T, d), rand(B, Hkv, T, d)
        cnt = _dev(nodes, gpu)
        at, seen = ms.tree_mask(_dev(parents, gpu), lens, counts=cnt, window=W, sinks=S)
        qr = ms.cache_append(cache, table, lens, k, v, q=q, inv_freq=freq, counts=cnt, positions=many(at), axis=axis)
        total = lens + cnt
        out, lse = ms.cache_tree_attn(cache, table, total, qr, seen, positions=at, counts=cnt, window=W, sinks=S)
        # every node against a cache of its own path
        for b in range(B):
            for t in (0, int(nodes[b]) - 1):
                line, u = [], t
                while u >= 0:
                    line.append(u)
                    u = int(parents[b, u])
                path = told[b] + [(k[b, :, u], v[b, :, u]) for u in line[::-1]]
                n = len(path)
                kk, vv = (torch.stack([x[i] for x in path], 1)[None] for i in (0, 1))
                kk, _ = ms.rotate(kk.contiguous(), None, many(torch.arange(n, dtype=I32, device=gpu)[None]), freq, axis=axis)
                i = torch.arange(n, device=gpu)
                sees = (n - 1 - i < W) | (i < S)
                G = Hq // Hkv
                z = (qr[b, :, t].double().view(Hkv, G, d) @ kk[0].double().transpose(1, 2).contiguous()) * d ** -0.5
                p = torch.softmax(z.masked_fill(~sees, -np.inf), -1)
                want = (p @ vv[0].double()).view(Hq, d)
                err = (out[b, :, t].double() - want).abs()
                # The cache's 8-bit rounding apart: a value is off by at most 2^-4 of itself (2^-3 where it moved to a larger
                # scale), evenly spread 0.036 of it; so is a key, which moves a logit of unit-normal rows by about 0.036 and
                # each weight by as much: 0.05 of the norm together, and 2.5 times that is allowed; one element by 2^-3 of
                # the largest value (below 4.8) itself
                assert float(err.max()) < 0.6 and float(err.norm() / want.norm()) < 0.13, (step, b, t)
        paths, kept = np.zeros((B, T), np.int64), []
        for b in range(B):
            line, u = [], int(rng.integers(0, nodes[b]))
            while u >= 0:
                line.append(u)
                u = int(parents[b, u])
            paths[b, :len(line)] = line[::-1]
            kept.append(len(line))
            told[b] += [(k[b, :, u], v[b, :, u]) for u in line[::-1]]
        ms.cache_keep(cache, table, total, _dev(paths, gpu), _dev(np.array(kept), gpu), counts=cnt)
        lens = lens + _dev(np.array(kept), gpu)
        assert lens.tolist() == [len(x) for x in told]
        # what the cache holds for each token is its key and value, rounded to e4m3 at most twice
        kc, vc, ks, vs = _host(cache)
        for b in range(B):
            entries = table[b].cpu().numpy()
            n = len(told[b])
            vv = torch.stack([x[1] for x in told[b]], 1).double().cpu().numpy()
            for h in range(Hkv):
                _, got, have = OC.gather(kc, vc, ks, vs, entries[None], n, 0, h)
                assert have.all()
                assert (np.abs(got - vv[h]) <= 2.0 ** -3 * np.abs(vv[h]) + 2.0 ** -9 * 2.0 ** -6).all(), (step, b, h)
    table, lens, refs, _ = ms.cache_fork(cache, table, lens, refs, torch.tensor([-1], dtype=I32, device=gpu))
    assert not refs.any() and (table == -1).all() and lens.tolist() == [0]


def _attends(out, lse, q, want, lens):
    """Within the bound of the attention's roundings (oracle/tree.py, oracle/cache.py)."""
    ro, eo, rl = want
    assert (np.abs(to_f64(out.contiguous().cpu()) - ro) <= eo).all()
    gl = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(gl), np.isneginf(rl))
    d, fine = q.shape[3], np.isfinite(rl)
    reach = 8.0 * max(1.0, float(q.double().abs().max())) * np.sqrt(d)
    assert np.abs(gl[fine] - rl[fine]).max() <= OW.lse_bound(int(lens.max()), d, reach)


@pytest.mark.parametrize("Hq,Hkv,d,T,axes,W,S", [(4, 2, 64, 12, 1, 90, 4), (8, 2, 128, 70, 3, 0, 0), (4, 4, 64, 9, 2, 33, 0)])
def test_every_step_of_speculative_decoding(gpu, Hq, Hkv, d, T, axes, W, S):
    """The loop of all operators, each step's result against the oracle on what the cache held before it: forks, moves of
    kept tokens and masks equal, attention within the bound of its roundings on the codes that the cache holds, and a token
    appended behind the accepted ones attends to them as the oracle's does."""
    print(f"every step Hq{Hq} Hkv{Hkv} d{d} T{T} axes{axes} W{W} S{S}", flush=True)
    B, pages, width = 3, 90, 9
    rng = np.random.default_rng(T)
    g = torch.Generator().manual_seed(T)
    rand = lambda *s: torch.randn(s, generator=g).to(BF).to(gpu)  # noqa: E731
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).float().to(gpu)
    axis = (torch.arange(d // 2) % axes).to(I32).to(gpu)
    many = lambda at: (at[None] * torch.arange(1, axes + 1, dtype=I32, device=gpu)[:, None, None]).contiguous()  # noqa: E731
    cache = _pool(19, pages, Hkv, d, gpu)
    table = torch.full((B, width), -1, dtype=I32, device=gpu)
    lens, refs = torch.zeros(B, dtype=I32, device=gpu), torch.zeros(pages, dtype=I32, device=gpu)

    def fork(src, room):
        got = _fork(gpu, cache, table.cpu().numpy(), lens.tolist(), refs.cpu().numpy(), src, room)
        assert not got[3].any()
        return tuple(_dev(x, gpu) for x in got[:3])

    prompt = [60, 64, 117]
    table, lens, refs = fork([0, 1, 2], prompt)
    at, counts = torch.arange(117, dtype=I32, device=gpu).expand(B, 117), _dev(np.array(prompt), gpu)
    ms.cache_append(cache, table, lens, rand(B, Hkv, 117, d), rand(B, Hkv, 117, d), inv_freq=freq, counts=counts,
                    positions=many(at), axis=axis)
    lens = lens + counts
    for step, src in enumerate(([0, 1, 2], [2, 0, 2], [0, 1, 2], [1, 1, 0])):
        table, lens, refs = fork(src, [n + T + 1 for n in lens[list(src)].tolist()])
        parents = (np.sqrt(rng.random((B, T))) * (np.arange(T) + 1)).astype(np.int64) - 1
        nodes = rng.integers(1, T + 1, B)
        q, k, v, cnt = rand(B, Hq, T, d), rand(B, Hkv, T, d), rand(B, Hkv, T, d), _dev(nodes, gpu)
        gat, seen = ms.tree_mask(_dev(parents, gpu), lens, counts=cnt, window=W, sinks=S)
        both = [OT.mask(parents[b], int(lens[b]), int(nodes[b]), W, S) for b in range(B)]
        at, sees = np.stack([x[0] for x in both]), np.stack([x[1] for x in both])
        assert np.array_equal(gat.cpu().numpy(), at) and np.array_equal(seen.cpu().numpy(), OT.words(sees))
        qr = ms.cache_append(cache, table, lens, k, v, q=q, inv_freq=freq, counts=cnt, positions=many(gat), axis=axis)
        total = lens + cnt
        host, entries, n = _host(cache), table.cpu().numpy(), total.cpu().numpy()
        # the nodes are there: V's values to half a step of e4m3, and below its normal range of the page's scale
        for b in range(B):
            for h in range(Hkv):
                _, got, have = OC.gather(*host, entries[b][None], int(n[b]), 0, h)
                x = to_f64(v[b:b + 1, h:h + 1, :nodes[b]].contiguous().cpu())[0, 0]
                new = got[n[b] - nodes[b]:]
                assert have.all() and (np.abs(new - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * host[3][:, h].max()).all()
        out, lse = ms.cache_tree_attn(cache, table, total, qr, seen, positions=gat, counts=cnt, window=W, sinks=S)
        torch.cuda.synchronize()
        _attends(out, lse, qr, OT.attention(to_f64(qr.cpu()), *host, entries, n, sees, at, nodes, W, S, d ** -0.5), n)
        path, kept = np.zeros((B, T), np.int64), []
        for b in range(B):
            line, u = [], int(rng.integers(0, nodes[b]))
            while u >= 0:
                line.append(u)
                u = int(parents[b, u])
            path[b, :len(line)] = line[::-1]
            kept.append(len(line))
        _keep(gpu, Hkv, d, T, n, [int(x) for x in nodes], path, kept, table=entries, cache=cache)
        lens = lens + _dev(np.array(kept), gpu)
        # the next token, behind the accepted ones
        q1, k1, v1 = rand(B, Hq, 1, d), rand(B, Hkv, 1, d), rand(B, Hkv, 1, d)
        qr = ms.cache_append(cache, table, lens, k1, v1, q=q1, inv_freq=freq, positions=many(lens[:, None]), axis=axis)
        lens = lens + 1
        out, lse = ms.cache_attn(cache, table, lens, qr, window=W, sinks=S)
        torch.cuda.synchronize()
        n = lens.cpu().numpy()
        _attends(out, lse, qr, OC.attention(to_f64(qr.cpu()), *_host(cache), entries, n, W, S, d ** -0.5), n)
    got = _fork(gpu, cache, table.cpu().numpy(), lens.tolist(), refs.cpu().numpy(), [-1], None)
    assert not got[2].any() and (got[0] == -1).all()
