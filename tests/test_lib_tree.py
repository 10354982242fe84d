"""Host-side checks of the rotation by positions, the drafted trees and the moves in the cache: refusals before any launch
(fake pointers that are never dereferenced), workspace queries, and the oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import cache as OC
from oracle import pages as OP
from oracle import tree as OT
from oracle import window as OW

P16 = 4096


def _p(x):
    return None if x is None else ctypes.c_void_p(x)


def _tensor(h, n=100, d=64, data=P16, token=None, head=None, batch=None):
    token = d if token is None else token
    head = n * d if head is None else head
    return ms.Tensor(data, h * n * d if batch is None else batch, head, token)


def _message():
    return ms.lib().msparse_last_error().decode()


def _cache(**change):
    f = dict(k=P16, v=P16, k_scale=P16, v_scale=P16, page_table=P16, lens=P16, pages=10, width=4, batch=2, heads_kv=2,
             head_dim=64)
    f.update(change)
    return ms.CacheStruct(*(f[n] for n, _ in ms.CacheStruct._fields_))


CACHE_REFUSALS = [
    (dict(batch=0), -1), (dict(heads_kv=0), -1), (dict(head_dim=80), -2), (dict(pages=0), -1),
    (dict(width=0), -1), (dict(width=(1 << 24) + 1), -2), (dict(k=None), -1), (dict(v=P16 + 8), -1),
    (dict(k_scale=None), -1), (dict(v_scale=P16 + 2), -1), (dict(page_table=None), -1), (dict(lens=None), -1),
]


def _rotate(batch=2, tokens=100, hq=4, hkv=2, d=64, type=0, pos=None, q=None, k=None, qo=None, ko=None, keys=True):
    pos = pos or ms.PositionsStruct(P16, None, P16, 1)
    n = max(tokens, 1)
    t = lambda h, at: _tensor(h, n, data=at)  # noqa: E731
    return ms.lib().msparse_rotate(batch, tokens, hq, hkv, d, type, pos, 0, q or t(4, P16),
                                   (k or t(2, 2 * P16)) if keys else None, qo or t(4, 3 * P16),
                                   (ko or t(2, 4 * P16)) if keys else None, None)


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), -1), (dict(tokens=-1), -1), (dict(hq=0), -1), (dict(hkv=-1), -1), (dict(d=96), -2), (dict(type=2), -1),
    (dict(type=-1), -1), (dict(tokens=1 << 30), -2), (dict(batch=1 << 30), -2), (dict(hkv=0), -1), (dict(keys=False), -1),
    (dict(pos=ms.PositionsStruct(None, None, P16, 1)), -1), (dict(pos=ms.PositionsStruct(P16, None, None, 1)), -1),
    (dict(pos=ms.PositionsStruct(P16, None, P16, 0)), -1), (dict(pos=ms.PositionsStruct(P16, None, P16, 5)), -1),
    (dict(pos=ms.PositionsStruct(P16 + 2, None, P16, 1)), -1), (dict(pos=ms.PositionsStruct(P16, P16 + 1, P16, 1)), -1),
    (dict(q=_tensor(4, data=None)), -1), (dict(k=_tensor(2, data=P16 + 8)), -1), (dict(qo=_tensor(4, token=0)), -1),
    (dict(ko=_tensor(2, token=68)), -1), (dict(qo=_tensor(4, data=P16, token=128, head=12800, batch=51200)), -1),
    (dict(ko=_tensor(2, data=2 * P16, token=128, head=12800, batch=25600)), -1),
])
def test_rotate_refuses(change, status):
    assert _rotate(**change) == status, _message()


def test_rotate_of_nothing():
    assert _rotate(tokens=0) == 0
    assert _rotate(tokens=0, hkv=0, keys=False) == 0


def test_append_at_refuses():
    c, n, L = _cache(), 5, ms.lib()
    pos = ms.PositionsStruct(P16, P16, P16, 3)

    def append(c=c, tokens=n, p=pos, k=None, counts=None):
        kv = _tensor(2, n)
        return L.msparse_cache_append_at(c, 4, tokens, _tensor(4, n), k or kv, kv, _tensor(4, n, data=2 * P16), p, counts,
                                         None)

    assert append(p=None) == -1 and "positions" in _message()
    for bad in ((None, None, P16, 1), (P16, None, None, 1), (P16, None, P16, 0), (P16, None, P16, 5), (P16 + 1, None, P16, 1)):
        assert append(p=ms.PositionsStruct(*bad)) == -1
    assert append(tokens=-1) == -1 and append(k=_tensor(2, n, token=4)) == -1 and append(counts=_p(P16 + 2)) == -1
    assert append(tokens=0) == 0
    for change, status in CACHE_REFUSALS:
        assert append(c=_cache(**change)) == status, (change, _message())


def test_tree_mask_refuses():
    L = ms.lib()

    def mask(batch=2, tokens=5, parents=P16, lens=P16, counts=None, window=0, sinks=0, at=P16, seen=P16):
        return L.msparse_tree_mask(batch, tokens, _p(parents), _p(lens), _p(counts), window, sinks, _p(at), _p(seen), None)

    for change, status in ((dict(batch=0), -1), (dict(tokens=-1), -1), (dict(tokens=1025), -2), (dict(batch=(1 << 22) + 1), -2),
                           (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(parents=None), -1), (dict(lens=None), -1),
                           (dict(at=None), -1), (dict(seen=None), -1), (dict(seen=P16 + 2), -1), (dict(counts=P16 + 1), -1)):
        assert mask(**change) == status, (change, _message())
    assert mask(tokens=0, parents=None) == 0


def test_tree_attn_refuses():
    L, n = ms.lib(), 5
    big = _cache(width=1000)

    def attn(c=big, tokens=n, window=0, sinks=0, scale=0.0, q=None, seen=P16, at=None, counts=None, out=None, lse=None, ws=P16,
             room=1 << 40):
        return L.msparse_cache_tree_attn(c, 4, tokens, window, sinks, scale, q or _tensor(4, n), _p(seen), _p(at), _p(counts),
                                         out or _tensor(4, n, data=2 * P16), _p(lse), _p(ws), room, None)

    need = L.msparse_cache_tree_attn_workspace(big, 4, n)
    assert need > 0 and L.msparse_cache_tree_attn_workspace(_cache(width=4), 4, n) == 0
    assert L.msparse_cache_tree_attn_workspace(big, 4, 1025) == 0
    for change, status in ((dict(tokens=1025), -2), (dict(tokens=-1), -1), (dict(window=-1), -1), (dict(sinks=-1), -1),
                           (dict(scale=float("nan")), -1), (dict(seen=None), -1), (dict(seen=P16 + 2), -1),
                           (dict(window=4), -1), (dict(window=4, at=P16 + 1), -1), (dict(counts=P16 + 2), -1),
                           (dict(q=_tensor(4, n, data=None)), -1), (dict(out=_tensor(4, n, head=0)), -1),
                           (dict(lse=P16 + 4), -1), (dict(room=need - 1), -4), (dict(ws=None), -4), (dict(ws=P16 + 8), -1)):
        assert attn(**change) == status, (change, _message())
    assert attn(tokens=0) == 0
    for change, status in CACHE_REFUSALS:
        assert attn(c=_cache(**change)) == status, (change, _message())


def test_keep_refuses():
    L = ms.lib()

    def keep(c=None, tokens=5, path=P16, kept=P16, counts=None):
        return L.msparse_cache_keep(c or _cache(), tokens, _p(path), _p(kept), _p(counts), None)

    for change, status in ((dict(tokens=-1), -1), (dict(path=None), -1), (dict(kept=None), -1), (dict(path=P16 + 2), -1),
                           (dict(kept=P16 + 1), -1), (dict(counts=P16 + 2), -1),
                           (dict(c=_cache(batch=1 << 22, heads_kv=2), tokens=1), -2)):
        assert keep(**change) == status, (change, _message())
    assert keep(tokens=0, path=None) == 0
    assert L.msparse_cache_keep(None, 5, _p(P16), _p(P16), None, None) == -1
    for change, status in CACHE_REFUSALS:
        assert keep(c=_cache(**change)) == status, (change, _message())


def test_fork_refuses():
    L, c = ms.lib(), _cache()
    need = L.msparse_cache_fork_workspace(c, 3)
    assert need > 0

    def fork(c=c, n=3, src=P16, room=None, refs=P16, refs_out=P16, table=2 * P16, lens=2 * P16, missing=P16, ws=P16, size=need):
        return L.msparse_cache_fork(c, n, *(_p(x) for x in (src, room, refs, refs_out, table, lens, missing, ws)), size, None)

    for change, status in ((dict(n=0), -1), (dict(n=-1), -1), (dict(n=65537), -2), (dict(src=None), -1), (dict(refs=None), -1),
                           (dict(refs_out=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(missing=None), -1),
                           (dict(src=P16 + 2), -1), (dict(room=P16 + 1), -1), (dict(table=P16), -1), (dict(lens=P16), -1),
                           (dict(ws=None), -4), (dict(size=need - 1), -4), (dict(ws=P16 + 4), -1),
                           (dict(c=_cache(batch=65537)), -2)):
        assert fork(**change) == status, (change, _message())
    assert L.msparse_cache_fork_workspace(c, 0) == 0 and L.msparse_cache_fork_workspace(c, 65537) == 0
    for change, status in CACHE_REFUSALS:
        assert fork(c=_cache(**change)) == status, (change, _message())


def test_fork_refuses_shared_memory():
    """What a call writes shares no word with what it reads or else writes, but refs_out with refs."""
    L, n = ms.lib(), 3
    c = _cache(page_table=1 << 16, lens=2 << 16)
    need = L.msparse_cache_fork_workspace(c, n)
    at = dict(src=3 << 16, room=4 << 16, refs=5 << 16, refs_out=6 << 16, table=7 << 16, lens=8 << 16, missing=9 << 16, ws=10 << 16)
    words = dict(src=n, room=n, refs=10, refs_out=10, table=4 * n, lens=n, missing=n, ws=need // 4, page_table=8, old_lens=2)
    everything = dict(at, page_table=1 << 16, old_lens=2 << 16)
    names = dict(refs_out="refs_out", table="page_table_out", lens="lens_out", missing="missing", ws="workspace")
    for out, name in names.items():
        for other in everything:
            if other == out:
                continue
            for off in (0, 4 * words[other] - 4, 4 - 4 * words[out]):   # the same, its last word, this one's last word
                if (out, other, off) in (("refs_out", "refs", 0),) or (out == "ws" and off % 16):
                    continue
                args = dict(at, **{out: everything[other] + off})
                assert L.msparse_cache_fork(c, n, *(_p(x) for x in args.values()), need, None) == -1, (out, other, off)
                assert name in _message() and "share memory" in _message(), (out, other, off, _message())
    for other in ("src", "room", "lens", "missing"):   # counts in their place, and another array there too
        args = dict(at, refs=at["refs_out"], **{other: at["refs_out"]})
        assert L.msparse_cache_fork(c, n, *(_p(x) for x in args.values()), need, None) == -1 and "share" in _message(), other


def test_binding_refuses_host_tensors_shapes_and_types():
    bf = torch.bfloat16
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q = torch.zeros((1, 2, 8, 64), dtype=bf)
    cache = ms.make_cache(2, 2, 64, "cpu")
    for call in (lambda: ms.rotate(q, q, i32(1, 1, 8), torch.zeros(32)),
                 lambda: ms.tree_mask(i32(1, 8), i32(1)),
                 lambda: ms.cache_append(cache, i32(1, 1), i32(1), q, q, inv_freq=torch.zeros(32), positions=i32(1, 8)),
                 lambda: ms.cache_tree_attn(cache, i32(1, 1), i32(1), q, i32(1, 8, 1)),
                 lambda: ms.cache_keep(cache, i32(1, 1), i32(1), i32(1, 8), i32(1)),
                 lambda: ms.cache_fork(cache, i32(1, 1), i32(1), i32(2), i32(3))):
        with pytest.raises(ms.MsparseError):
            call()


# ---------------------------------------------------------------- the oracle's pins
def test_oracle_rotation_of_one_axis_is_the_caches():
    rng = np.random.default_rng(0)
    x, pos, f = rng.standard_normal((6, 64)), rng.integers(0, 1000, (1, 6)), 10000.0 ** (-np.arange(32) / 32)
    y = OT.rotate(x, pos, f)
    assert np.array_equal(y, OC.rotate(x, pos[0], f))
    assert np.allclose(OT.rotate(y, pos, f, inverse=True), x, atol=1e-12)
    # two axes: each pair goes by its own; none: it stays
    two = np.concatenate([pos, pos[:, ::-1]])
    z = OT.rotate(x, two, f, np.array([0, 1] * 15 + [2, -1]))
    for i, p in ((0, pos[0]), (1, pos[0, ::-1])):
        c = (x[:, i] + 1j * x[:, 32 + i]) * np.exp(1j * p * f[i])
        assert np.allclose(z[:, i], c.real) and np.allclose(z[:, 32 + i], c.imag)
    assert np.array_equal(z[:, [30, 31, 62, 63]], x[:, [30, 31, 62, 63]])


def test_oracle_chain_mask_is_the_windows():
    for n, T, W, S in ((0, 9, 3, 2), (5, 7, 0, 0), (20, 6, 4, 22), (3, 5, 1, 0)):
        at, sees = OT.mask(np.arange(T) - 1, n, T, W, S)
        full = OW.mask(n + T, W, S)
        assert np.array_equal(at, n + np.arange(T)) and np.array_equal(sees, full[n:, n:])
    at, sees = OT.mask([-1, 0, 0, 2, 9, 1], 10, 5)
    assert at.tolist() == [10, 11, 11, 12, 10, 10]
    assert [np.flatnonzero(r).tolist() for r in sees] == [[0], [0, 1], [0, 2], [0, 2, 3], [4], []]
    w = OT.words(np.eye(40, dtype=bool))
    assert w.shape == (40, 2) and w[31].tolist() == [-2 ** 31, 0] and w[39].tolist() == [0, 128]


def test_oracle_tree_attention_of_a_chain_is_the_caches():
    rng = np.random.default_rng(1)
    d, n, T = 8, 70, 6
    k, v = rng.integers(0, 127, (2, 1, 64, d)).astype(np.uint8), rng.integers(0, 127, (2, 1, d, 64)).astype(np.uint8)
    ks, vs = np.full((2, 1), 2.0 ** -7), np.full((2, 1), 2.0 ** -7)
    q, table, lens = rng.standard_normal((1, 2, T, d)), np.array([[1, 0]]), [n + T]
    for W, S in ((0, 0), (9, 3)):
        at, sees = OT.mask(np.arange(T) - 1, n, T, W, S)
        a = OT.attention(q, k, v, ks, vs, table, lens, sees[None], at[None], [T], W, S, 0.3)
        b = OC.attention(q, k, v, ks, vs, table, lens, W, S, 0.3)
        for x, y in zip(a, b):
            assert np.allclose(x, y)


def test_oracle_keep_moves_values():
    """Within one page codes move as they are; between pages of other scales the values do."""
    rng = np.random.default_rng(2)
    k, v = rng.integers(8, 0x70, (3, 2, 64, 8)).astype(np.uint8), rng.integers(8, 0x70, (3, 2, 8, 64)).astype(np.uint8)
    ks, vs = np.array([[1.0, 2.0], [4.0, 0.25], [1.0, 1.0]]), np.array([[0.5, 2.0], [1.0, 8.0], [1.0, 1.0]])
    table, path = np.array([[1, 0]]), np.array([[1, 5, 9, 0]])
    before = [OC.gather(k, v, ks, vs, table, 75, 0, h)[:2] for h in range(2)]
    old = k.copy()
    OP.keep(k, v, ks, vs, table, [75], path, [3], [15])   # nodes at 60 .. 74: 60, 61, 62 take 61, 65, 69
    after = [OC.gather(k, v, ks, vs, table, 63, 0, h)[:2] for h in range(2)]
    at = list(range(60)) + [61, 65, 69]
    for x, y in zip(before, after):
        for a, b in zip(x, y):
            assert np.abs(a[at] - b).max() <= 2.0 ** -3 * np.abs(b).max()
            fine = np.abs(a[at]) >= 2.0 ** -6 * 8
            assert np.array_equal(a[at][fine], b[fine])
    assert np.array_equal(k[2], old[2]) and np.array_equal(k[0], old[0])
    assert (k[1, :, 63] == old[1, :, 63]).all()


def test_oracle_fork_by_hand():
    table = np.array([[4, 2, 6, -1], [1, 3, -1, -1]])
    refs = np.array([1, 1, 2, 1, 1, 0, 1, 0])
    got = OP.fork(table, [100, 128], refs, [0, 0, 1, -1], [300, 0, 200, 10], 8)
    # row 0 keeps 4, 2 and 6, and wants one more; row 1 shares 4 and copies 2; row 2 keeps both and wants two; row 3 one
    assert got[0].tolist() == [[4, 2, 6, 5], [4, 7, -1, -1], [1, 3, -1, -1], [-1] * 4]
    assert got[1].tolist() == [100, 100, 128, 0] and got[3].tolist() == [0, 0, 2, 1]
    assert got[2].tolist() == [1, 1, 2, 1, 2, 1, 1, 1] and got[4] == [(2, 7)]
    # pages that another table holds too: the partly filled one stays with the first, the second one's copy is its own
    got = OP.fork(np.array([[4, 2, -1]]), [100], np.array([0, 0, 2, 0, 2, 0]), [0, 0], None, 6)
    assert got[0].tolist() == [[4, 2, -1], [4, 0, -1]] and got[2].tolist() == [1, 0, 2, 0, 3, 0] and got[4] == [(2, 0)]
