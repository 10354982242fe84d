"""The paged cache at the ends of its ranges: sequences longer than their tables, rows that are not finite, tables
whose pages pass 32 bits together.  Against the fp64 oracle as in test_gpu_cache.py."""
import pytest
import torch

import paper_2510_18830_amd as ms
from tests.test_gpu_cache import _attn_check, _filled, _randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,d,T,width,W,S", [
    (4, 2, 64, 3, 5, 0, 0), (4, 2, 64, 3, 5, 70, 5), (4, 2, 64, 1, 5, 40, 0),
    (4, 2, 128, 3, 12, 0, 0), (4, 2, 128, 3, 12, 100, 70), (4, 2, 128, 1, 12, 40, 0), (4, 1, 64, 9, 12, 75, 0),
    (4, 1, 128, 40, 3, 0, 0), (4, 1, 64, 40, 12, 0, 0), (4, 1, 128, 40, 12, 90, 3), (2, 2, 64, 200, 12, 33, 0),
])
def test_attn_past_the_table(gpu, Hq, Hkv, d, T, width, W, S):
    """Rows keep the positions of the whole length: those past the table see what their window and the sinks leave of
    the tokens that have a page, the rows before them what their own positions see."""
    print(f"past the table Hq{Hq} Hkv{Hkv} d{d} T{T} width{width} W{W} S{S}", flush=True)
    room = 64 * width
    cache, table, _ = _filled(T + width, [room] * 6, Hkv, d, gpu)
    lens = [room, room + 1, room + 5, room + 64, room + T - 1, room + 1000]
    q = _randn(1, (len(lens), Hq, T, d), gpu)
    out, lse = ms.cache_attn(cache, table, torch.tensor(lens, dtype=torch.int32, device=gpu), q, window=W, sinks=S)
    torch.cuda.synchronize()
    _attn_check(q, out, lse, cache, table, lens, W, S)


@pytest.mark.parametrize("W,S", [(0, 0), (50, 0), (50, 7), (2 ** 31 - 1, 3)])
@pytest.mark.parametrize("d,T", [(64, 1), (128, 3), (64, 70)])
def test_attn_lengths_up_to_32_bits(gpu, d, T, W, S):
    """A far length sees what any length past the window sees: all tokens that have a page, the sinks', or none."""
    cache, table, _ = _filled(31, [640] * 4, 2, d, gpu)
    q = _randn(1, (1, 4, T, d), gpu).expand(4, 4, T, d).contiguous()
    got = []
    for n in (100000, 2 ** 31 - 64):
        lens = torch.full((4,), n, dtype=torch.int32, device=gpu)
        got.append(ms.cache_attn(cache, table, lens, q, window=W, sinks=S))
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert not torch.isneginf(got[1][1]).any() if W != 50 or S else torch.isneginf(got[1][1]).all()


@pytest.mark.parametrize("d,T,lens", [(64, 1, [40, 700, 9000]), (128, 1, [40, 700, 9000]), (128, 5, [40, 3000]),
                                      (64, 70, [200, 3000]), (128, 600, [1500])])
def test_attn_queries_that_are_not_finite(gpu, d, T, lens):
    """A NaN in a query: its row's out and lse are NaN (not the -inf of a row without a key), the others' unchanged."""
    cache, table, L = _filled(37, lens, 2, d, gpu)
    q = _randn(1, (len(lens), 4, T, d), gpu)
    want = ms.cache_attn(cache, table, L, q)
    bad = torch.zeros((len(lens), 4, T), dtype=torch.bool, device=gpu)
    bad[:, 1, T - 1] = bad[0, 2, 0] = True
    q[bad] = torch.where(torch.arange(d, device=gpu) == 5, float("nan"), 1.0).to(q.dtype)
    out, lse = ms.cache_attn(cache, table, L, q)
    torch.cuda.synchronize()
    assert torch.isnan(lse[bad]).all() and torch.isnan(out[bad]).all()
    assert torch.equal(out[~bad], want[0][~bad]) and torch.equal(lse[~bad], want[1][~bad])


def test_attn_pages_beyond_32_bits(gpu):
    """260 sequences of 2^30 tokens: more than 2^32 pages together, of which each sequence's table holds seven.  The
    result is that of the seven pages alone."""
    B, Hkv, d, width, held = 260, 1, 64, 1 << 24, 7
    cache, table, L = _filled(41, [64 * held] * B, Hkv, d, gpu)
    wide = torch.full((B, width), -1, dtype=torch.int32, device=gpu)
    for i, at in enumerate((0, 3, 70000, 1 << 22, (1 << 23) + 5, (1 << 24) - 9, (1 << 24) - 1)):
        wide[:, at] = table[:, i]
    lens = torch.full((B,), 64 * width, dtype=torch.int32, device=gpu)
    q = _randn(1, (B, 4, 1, d), gpu)
    torch.cuda.synchronize()
    print("tables made", flush=True)
    out, lse = ms.cache_attn(cache, wide, lens, q)
    torch.cuda.synchronize()
    _attn_check(q, out, lse, cache, table, [64 * held] * B, 0, 0)
