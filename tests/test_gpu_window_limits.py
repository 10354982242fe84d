"""Window attention on the largest grids, and packed documents whose grids are made from the tensors' rows.  Against the
fp64 oracle as in test_gpu_window.py."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from tests.test_gpu_window import _check, _inputs

pytestmark = pytest.mark.gpu


def test_window_sums_of_many_groups(gpu):
    """2^19 sequences and heads whose sinks leave partial sums (a workspace of 137 GB): all get their gradients."""
    torch.cuda.empty_cache()
    B, H, n, d, W, S = 65536, 8, 2, 128, 1, 1
    one = _inputs(7, 1, H, H, n, d, gpu)
    q, k, v, do = (t.expand(B, H, n, d) for t in one)
    win = ms.make_window(B, n, H, H, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = [torch.full((B, H, n, d), 7.0, dtype=torch.bfloat16, device=gpu) for _ in range(3)]
    room = torch.empty(ms.window_bwd_workspace_bytes(win), dtype=torch.uint8, device=gpu)
    print(f"workspace {room.numel() / 1e9:.0f} GB", flush=True)
    ms.window_bwd(win, q, k, v, out, do, lse, dq=grads[0], dk=grads[1], dv=grads[2], workspace=room)
    torch.cuda.synchronize()
    del room
    torch.cuda.empty_cache()
    _check(*one, out[:1], lse[:1], [g[:1] for g in grads], W, S, d ** -0.5)
    for g in grads:
        assert (g == g[:1]).all()


def _packed(seed, lens, before, after, Hq, Hkv, d, gpu):
    """Documents of `lens` rows, rows of none before and behind them (NaN), and their starts."""
    starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32) + before
    total = int(starts[-1]) + after
    x = _inputs(seed, 1, Hq, Hkv, total, d, gpu)
    for t in x:
        t[:, :, :before] = float("nan")
        t[:, :, total - after:] = float("nan")
    return x, starts, total


def _run(win, x, st):
    q, k, v, do = x
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:3], 7.0, device=q.device)
    grads = [torch.full_like(t, 7.0) for t in (q, k, v)]
    ms.window_fwd(win, q, k, v, starts=st, out=out, lse=lse)
    ms.window_bwd(win, q, k, v, out, do, lse, starts=st, dq=grads[0], dk=grads[1], dv=grads[2])
    torch.cuda.synchronize()
    return out, lse, grads


def _lens(seed, docs, short, long):
    """Documents of up to `short` rows, some empty, and the long ones among them."""
    g = np.random.default_rng(seed)
    lens = [int(n) for n in g.integers(0, short + 1, docs)]
    for n in long:
        lens[int(g.integers(0, docs))] = n
    return lens


@pytest.mark.parametrize("docs,short,long,Hq,Hkv,d,W,S", [
    (40, 60, [2500], 4, 2, 64, 100, 4), (40, 60, [2500], 4, 1, 128, 100, 4), (60, 5, [1300, 700], 2, 2, 128, 0, 0),
    (90, 30, [1700], 3, 1, 64, 64, 130), (90, 30, [1700], 2, 1, 128, 300, 500), (30, 200, [], 8, 2, 64, 16, 1),
    (5000, 6, [900, 77], 2, 1, 64, 33, 2), (4200, 3, [400], 1, 1, 128, 0, 0), (65, 1, [600], 1, 1, 64, 1, 1),
    (20, 130, [3000], 14, 2, 128, 1, 3), (64, 40, [2049, 2048, 65], 6, 2, 64, 127, 64),
])
def test_window_packed_by_rows(gpu, docs, short, long, Hq, Hkv, d, W, S):
    """Many short documents around few long ones, the longest not known: grids by the tensors' rows."""
    print(f"packed {docs} docs up to {short}, {long}, Hq{Hq} Hkv{Hkv} d{d} W{W} S{S}", flush=True)
    lens = _lens(docs + W, docs, short, long)
    x, starts, total = _packed(docs, lens, 5, 9, Hq, Hkv, d, gpu)
    win = ms.make_window(docs, total, Hq, Hkv, d, W, S, tokens=total)
    st = starts.to(gpu)
    out, lse, grads = _run(win, x, st)
    again = _run(win, x, st)
    for a, b in zip((out, lse, *grads), (*again[:2], *again[2])):
        assert torch.equal(a, b)
    order = sorted(range(docs), key=lambda b: -lens[b])
    for b in sorted(set(order[:4] + order[docs // 2:docs // 2 + 8] + [0, 1, 63, 64, docs - 2, docs - 1]) & set(range(docs))):
        if lens[b]:
            _check(*x, out, lse, grads, W, S, d ** -0.5, int(starts[b]), lens[b])
    for t in (out, lse, *grads):
        assert (t[:, :, :5] == 7).all() and (t[:, :, total - 9:] == 7).all()
        assert torch.isfinite(t).all()


@pytest.mark.parametrize("d", [64, 128])
def test_window_packed_by_rows_on_large_grids(gpu, d):
    """100 documents in 64K rows, one of them half: more workgroups than the kernels for small grids take."""
    Hq, Hkv, W, S = 16, 2, 200, 4
    lens = _lens(d, 100, 640, [])
    lens[37] = 65536 - sum(lens) + lens[37]
    x, starts, total = _packed(3, lens, 0, 0, Hq, Hkv, d, gpu)
    win = ms.make_window(100, total, Hq, Hkv, d, W, S, tokens=total)
    st = starts.to(gpu)
    out, lse, grads = _run(win, x, st)
    for b in (0, 36, 38, 70, 99):
        if lens[b]:
            _check(*x, out, lse, grads, W, S, d ** -0.5, int(starts[b]), lens[b])
    at, n = int(starts[37]), lens[37]
    alone = [t[:, :, at:at + n].contiguous() for t in x]
    one = ms.make_window(1, n, Hq, Hkv, d, W, S)
    o1, l1 = ms.window_fwd(one, *alone[:3])
    g1 = ms.window_bwd(one, *alone[:3], o1, alone[3], l1)
    torch.cuda.synchronize()
    part = [t[:, :, at:at + n] for t in (out, lse, *grads)]
    assert torch.equal(part[0], o1) and torch.equal(part[1], l1) and torch.equal(part[2], g1[0])
    # keys past the sinks' group: the same walk.  Those within: chunks of other lengths, so fp32 sums in another order,
    # 8 heads x 512 tiles x 2 additions of 2^-24 of a partial sum, on both sides: 2^-10 of the largest, here taken to be
    # up to twice the largest result; and a step of bf16 between the two roundings.
    for a, b in zip(part[3:], g1[1:]):
        assert torch.equal(a[:, :, 128:], b[:, :, 128:])
        a, b = a[:, :, :128].double(), b[:, :, :128].double()
        assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 2.0 ** -9 * b.abs().max()).all()


def test_window_packed_by_rows_starts_are_cut(gpu):
    """Starts out of range or order read and write inside the tensors; a long document is cut to `seq` rows."""
    q, k, v, do = _inputs(3, 1, 2, 1, 2000, 64, gpu)
    pad = [40000] * 60
    for starts in ([-50, 1000, 5000] + pad, [1500, 20, 2000] + pad, [1999] * 30 + [0] * 33, [7, 1500, 2000] + [2000] * 60):
        print(starts[:3], flush=True)
        win = ms.make_window(62, 700, 2, 1, 64, 30, 2, tokens=2000)
        st = torch.tensor(starts, dtype=torch.int32, device=gpu)
        out, lse, grads = _run(win, (q, k, v, do), st)
    for at, n in ((7, 700), (1500, 500)):
        _check(q, k, v, do, out, lse, grads, 30, 2, 0.125, at, n)
    for t in (out, lse, *grads):
        assert (t[:, :, :7] == 7).all() and (t[:, :, 707:1500] == 7).all()


def test_window_packed_by_rows_captured(gpu):
    """Forward and backward in one graph, replayed on other documents of the same tensors."""
    Hq, Hkv, d, docs, total = 4, 2, 64, 50, 1500
    win = ms.make_window(docs, total, Hq, Hkv, d, 60, 3, tokens=total)
    x = _inputs(5, 1, Hq, Hkv, total, d, gpu)
    st = torch.zeros(docs + 1, dtype=torch.int32, device=gpu)

    def fill(seed):
        cuts = np.sort(np.random.default_rng(seed).integers(0, total + 1, docs - 1))
        st.copy_(torch.tensor([0, *cuts.tolist(), total], dtype=torch.int32))

    def step():
        out, lse = ms.window_fwd(win, *x[:3], starts=st)
        return (out, lse) + ms.window_bwd(win, *x[:3], out, x[3], lse, starts=st)

    fill(1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (2, 3, 4):
        fill(seed)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("W,S", [(0, 0), (50, 3)])
def test_window_packed_longest_beyond_the_rows(gpu, W, S):
    """`seq` of 2^30, 128 heads on one: the walks (2^31 tiles by that length) are those of the tensors' rows."""
    lens, d = [200, 0, 100], 64
    x, starts, total = _packed(11, lens, 0, 0, 128, 1, d, gpu)
    st = starts.to(gpu)
    want = _run(ms.make_window(3, total, 128, 1, d, W, S, tokens=total), x, st)
    got = _run(ms.make_window(3, 1 << 30, 128, 1, d, W, S, tokens=total), x, st)
    for a, b in zip((*got[:2], *got[2]), (*want[:2], *want[2])):
        assert torch.equal(a, b)
    _check(*x, *got, W, S, d ** -0.5, 200, 100)
