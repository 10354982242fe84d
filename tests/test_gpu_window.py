"""Attention with a sliding window and sinks (window_fwd, window_bwd) against the
fp64 oracle, element by element within the bounds that the roundings to bf16
allow (oracle/window.py), and gradients against differences of the oracle's
forward.  Lengths, windows and sinks around the tiles' borders of 32, 64 and 128."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import window as OW
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu


def _make(seed, rows, heads, n, d, gpu, sharp=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, heads, n, d), generator=g) * sharp
    return x.to(torch.bfloat16).to(gpu)


def _inputs(seed, rows, Hq, Hkv, n, d, gpu, sharp=1.0):
    q, k = _make(seed, rows, Hq, n, d, gpu, sharp), _make(seed + 1, rows, Hkv, n, d, gpu, sharp)
    return q, k, _make(seed + 2, rows, Hkv, n, d, gpu), _make(seed + 3, rows, Hq, n, d, gpu)


def _within(name, got, ref, bound):
    err = np.abs(to_f64(got.contiguous().cpu()) - ref)
    assert np.isfinite(err).all(), name
    over = err - bound
    at = np.unravel_index(np.argmax(over), over.shape)
    assert over[at] <= 0, f"{name} off by {err[at]:.3e} at {at}, bound {bound[at]:.3e}"


def _check(q, k, v, do, out, lse, grads, W, S, scale, at=0, n=None):
    """One sequence: rows at .. at + n - 1 of batch entry 0."""
    n = q.shape[2] if n is None else n
    f = [to_f64(t[0, :, at:at + n].contiguous().cpu()) for t in (q, k, v, do)]
    d = q.shape[3]
    ro, eo, rl, reach = OW.sequence_fwd(f[0], f[1], f[2], W, S, scale)
    _within("out", out[0, :, at:at + n], ro, eo)
    el = np.abs(lse[0, :, at:at + n].double().cpu().numpy() - rl)
    assert el.max() <= OW.lse_bound(n, d, reach), f"lse off by {el.max():.3e}"
    if grads is None:
        return
    for name, got, (ref, bound) in zip(("dq", "dk", "dv"), grads, OW.sequence_bwd(*f, W, S, scale)):
        _within(name, got[0, :, at:at + n], ref, bound)


CASES = [  # Hq, Hkv, n, d, window, sinks
    (1, 1, 1, 64, 0, 0), (2, 1, 2, 128, 1, 1), (4, 2, 31, 64, 5, 2), (2, 2, 64, 128, 64, 0), (3, 1, 65, 64, 16, 3),
    (2, 1, 127, 128, 33, 0), (4, 1, 128, 64, 127, 1), (2, 1, 129, 128, 128, 64), (4, 2, 333, 64, 100, 7),
    (7, 1, 300, 128, 64, 65), (2, 1, 700, 128, 65, 4), (4, 2, 777, 64, 256, 4), (2, 1, 640, 64, 1, 0),
    (2, 1, 500, 128, 1, 130), (2, 2, 450, 64, 40, 449), (2, 1, 400, 128, 0, 5), (2, 1, 390, 64, 390, 5),
    (1, 1, 1500, 64, 70, 200), (2, 1, 1025, 128, 320, 16),
]


@pytest.mark.parametrize("Hq,Hkv,n,d,W,S", CASES)
def test_window_matches_oracle(gpu, Hq, Hkv, n, d, W, S):
    print(f"window Hq{Hq} Hkv{Hkv} n{n} d{d} W{W} S{S}", flush=True)
    q, k, v, do = _inputs(n, 1, Hq, Hkv, n, d, gpu)
    win = ms.make_window(1, n, Hq, Hkv, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = ms.window_bwd(win, q, k, v, out, do, lse)
    torch.cuda.synchronize()
    _check(q, k, v, do, out, lse, grads, W, S, d ** -0.5)


@pytest.mark.parametrize("sharp,scale", [(3.0, 0.0), (1.0, 0.7), (0.05, 0.0)])
def test_window_scales(gpu, sharp, scale):
    """Nearly one-hot rows, a scale of the caller's, nearly uniform rows."""
    q, k, v, do = _inputs(5, 1, 2, 1, 260, 64, gpu, sharp)
    win = ms.make_window(1, 260, 2, 1, 64, 90, 3, scale=scale)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = ms.window_bwd(win, q, k, v, out, do, lse)
    _check(q, k, v, do, out, lse, grads, 90, 3, scale or 0.125)


def test_window_batch_and_strides(gpu):
    """A batch as [B, N, H, d] memory, and keys that all heads share through stride 0."""
    B, Hq, Hkv, n, d = 3, 4, 2, 150, 64
    base = [_make(s, B, n, h, d, gpu) for s, h in ((1, Hq), (2, Hkv), (3, Hkv), (4, Hq))]
    q, k, v, do = (t.transpose(1, 2) for t in base)
    win = ms.make_window(B, n, Hq, Hkv, d, 40, 2)
    want = ms.window_fwd(win, *(t.contiguous() for t in (q, k, v)))
    out = torch.empty((B, n, Hq, d), dtype=torch.bfloat16, device=gpu).transpose(1, 2)
    got = ms.window_fwd(win, q, k, v, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    gw = ms.window_bwd(win, *(t.contiguous() for t in (q, k, v)), want[0], do.contiguous(), want[1])
    dq, dk, dv = (torch.empty((B, n, h, d), dtype=torch.bfloat16, device=gpu).transpose(1, 2) for h in (Hq, Hkv, Hkv))
    gg = ms.window_bwd(win, q, k, v, out, do, got[1], dq=dq, dk=dk, dv=dv)
    for a, b in zip(gg, gw):
        assert torch.equal(a, b)
    for b in range(B):
        _check(*(t[b:b + 1] for t in (q, k, v, do)), out[b:b + 1], got[1][b:b + 1], [x[b:b + 1] for x in gg], 40, 2,
               d ** -0.5)
    shared_k, shared_v = (t[:, :1].expand(B, Hkv, n, d) for t in (k, v))
    a = ms.window_fwd(win, q, shared_k, shared_v)
    b = ms.window_fwd(win, q, shared_k.contiguous(), shared_v.contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_window_packed(gpu):
    """Ragged documents, an empty one, rows before, behind and between none; a NaN in a row of no document."""
    lens, Hq, Hkv, d, W, S = [70, 0, 1, 129, 300, 64], 4, 2, 64, 50, 3
    starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32) + 5
    total = int(starts[-1]) + 9
    q, k, v, do = _inputs(9, 1, Hq, Hkv, total, d, gpu)
    for t in (q, k, v, do):
        t[:, :, :5] = float("nan")
        t[:, :, total - 9:] = float("nan")
    win = ms.make_window(len(lens), max(lens), Hq, Hkv, d, W, S, tokens=total)
    out = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:3], 7.0, device=gpu)
    dq, dk, dv = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    st = starts.to(gpu)
    ms.window_fwd(win, q, k, v, starts=st, out=out, lse=lse)
    ms.window_bwd(win, q, k, v, out, do, lse, starts=st, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    for at, n in zip(starts.tolist(), lens):
        if n:
            _check(q, k, v, do, out, lse, (dq, dk, dv), W, S, d ** -0.5, at, n)
    for t in (out, lse, dq, dk, dv):
        assert (t[:, :, :5] == 7).all() and (t[:, :, total - 9:] == 7).all()


def test_window_packed_starts_are_cut_to_the_tensors(gpu):
    """Starts out of range or order read and write inside the tensors; a long document is cut to `seq` rows."""
    q, k, v, do = _inputs(3, 1, 2, 1, 200, 64, gpu)
    for starts in ([-50, 100, 5000], [150, 20, 200], [0, 200, 200]):
        win = ms.make_window(2, 90, 2, 1, 64, 30, 2, tokens=200)
        st = torch.tensor(starts, dtype=torch.int32, device=gpu)
        out, lse = torch.full_like(q, 7.0), torch.full((1, 2, 200), 7.0, device=gpu)
        ms.window_fwd(win, q, k, v, starts=st, out=out, lse=lse)
        ms.window_bwd(win, q, k, v, out, do, lse, starts=st)
        torch.cuda.synchronize()
    _check(q, k, v, do, out, lse, None, 30, 2, 0.125, 0, 90)
    assert (out[:, :, 90:] == 7).all()


def test_window_equals_causal_when_it_reaches_everything(gpu):
    """window = 0, a window or sinks of the whole length: the same bits."""
    q, k, v, do = _inputs(21, 1, 2, 1, 210, 128, gpu)
    got = []
    for W, S in ((0, 0), (210, 0), (1000, 9), (3, 210), (0, 77)):
        win = ms.make_window(1, 210, 2, 1, 128, W, S)
        out, lse = ms.window_fwd(win, q, k, v)
        got.append((out, lse) + ms.window_bwd(win, q, k, v, out, do, lse))
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


def test_window_sinks_in_many_chunks(gpu):
    """Sink keys whose later rows are cut into many chunks, two pairs of key blocks, GQA; repeated calls agree."""
    Hq, Hkv, n, d, W, S = 4, 1, 5000, 64, 64, 150
    q, k, v, do = _inputs(31, 1, Hq, Hkv, n, d, gpu)
    win = ms.make_window(1, n, Hq, Hkv, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = ms.window_bwd(win, q, k, v, out, do, lse)
    again = ms.window_bwd(win, q, k, v, out, do, lse)
    for a, b in zip(grads, again):
        assert torch.equal(a, b)
    _check(q, k, v, do, out, lse, grads, W, S, d ** -0.5)


def test_window_gradients_against_differences(gpu):
    """The kernel's gradients along random directions against central differences of the oracle's loss."""
    Hq, Hkv, n, d, W, S = 2, 1, 140, 64, 30, 2
    q, k, v, do = _inputs(41, 1, Hq, Hkv, n, d, gpu)
    win = ms.make_window(1, n, Hq, Hkv, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = ms.window_bwd(win, q, k, v, out, do, lse)
    f = [to_f64(t[0].cpu()) for t in (q, k, v, do)]
    bounds = [b for _, b in OW.sequence_bwd(*f, W, S, d ** -0.5)]
    rng = np.random.default_rng(0)
    loss = lambda a, b, c: (OW.sequence_fwd(a, b, c, W, S, d ** -0.5)[0] * f[3]).sum()  # noqa: E731
    for x in range(3):
        step = rng.standard_normal(f[x].shape)
        eps = 1e-5
        plus, minus = [list(f[:3]) for _ in range(2)]
        plus[x], minus[x] = f[x] + eps * step, f[x] - eps * step
        diff = (loss(*plus) - loss(*minus)) / (2 * eps)
        got = (to_f64(grads[x][0].cpu()) * step).sum()
        assert abs(got - diff) <= (bounds[x] * np.abs(step)).sum() + 1e-6 * abs(diff)


def test_window_captured_and_replayed(gpu):
    """Forward and backward in one graph, replayed on other inputs with eager calls between."""
    Hq, Hkv, n, d = 4, 2, 300, 64
    win = ms.make_window(1, n, Hq, Hkv, d, 70, 5)
    static = list(_inputs(51, 1, Hq, Hkv, n, d, gpu))
    ws = torch.empty(ms.window_bwd_workspace_bytes(win), dtype=torch.uint8, device=gpu)

    def step():
        out, lse = ms.window_fwd(win, *static[:3])
        return (out, lse) + ms.window_bwd(win, *static[:3], out, static[3], lse, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (61, 62, 63):
        fresh = _inputs(seed, 1, Hq, Hkv, n, d, gpu)
        for a, b in zip(static, fresh):
            a.copy_(b)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_window_on_another_stream(gpu):
    q, k, v, do = _inputs(71, 1, 2, 1, 333, 128, gpu)
    win = ms.make_window(1, 333, 2, 1, 128, 64, 4)
    out, lse = ms.window_fwd(win, q, k, v)
    want = (out, lse) + ms.window_bwd(win, q, k, v, out, do, lse)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out, lse = ms.window_fwd(win, q, k, v, stream=s)
    got = (out, lse) + ms.window_bwd(win, q, k, v, out, do, lse, stream=s)
    s.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("B,Hq,Hkv,n,d,W,S", [
    (60, 8, 2, 129, 64, 50, 3), (40, 4, 4, 300, 128, 100, 7), (30, 8, 1, 260, 64, 0, 0), (24, 8, 4, 333, 128, 0, 0),
    (50, 4, 1, 500, 64, 5, 0), (16, 16, 2, 257, 128, 20, 130), (70, 7, 1, 70, 128, 3, 1),
])
def test_window_on_large_grids(gpu, B, Hq, Hkv, n, d, W, S):
    """More workgroups than the kernels for small grids take: the first, a middle and the last sequence."""
    q, k, v, do = _inputs(n, B, Hq, Hkv, n, d, gpu)
    win = ms.make_window(B, n, Hq, Hkv, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = ms.window_bwd(win, q, k, v, out, do, lse)
    torch.cuda.synchronize()
    for b in (0, B // 2, B - 1):
        at = slice(b, b + 1)
        _check(q[at], k[at], v[at], do[at], out[at], lse[at], [g[at] for g in grads], W, S, d ** -0.5)


@pytest.mark.parametrize("d", [64, 128])
def test_window_packed_on_large_grids(gpu, d):
    """Many documents, some empty, in tensors laid out as [tokens, heads, d]."""
    Hq, Hkv, W, S = 6, 2, 90, 4
    lens = (np.random.default_rng(d).integers(0, 420, 60) * (np.arange(60) % 7 != 3)).tolist()
    starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    total = int(starts[-1])
    q, k, v, do = (_make(s, 1, total, h, d, gpu).transpose(1, 2) for s, h in ((1, Hq), (2, Hkv), (3, Hkv), (4, Hq)))
    win = ms.make_window(len(lens), max(lens), Hq, Hkv, d, W, S, tokens=total)
    st = starts.to(gpu)
    out, lse = ms.window_fwd(win, q, k, v, starts=st)
    grads = ms.window_bwd(win, q, k, v, out, do, lse, starts=st)
    torch.cuda.synchronize()
    for b in (0, 1, 3, 30, 58, 59):
        if lens[b]:
            _check(q, k, v, do, out, lse, grads, W, S, d ** -0.5, int(starts[b]), lens[b])


@pytest.mark.parametrize("Hq,Hkv,n,d,W,S", [(2, 1, 2600, 64, 0, 0), (1, 1, 2100, 128, 600, 70), (8, 1, 1100, 128, 0, 0)])
def test_window_keys_in_several_walks(gpu, Hq, Hkv, n, d, W, S):
    """Few key groups with long walks over the rows, which are cut."""
    q, k, v, do = _inputs(n, 1, Hq, Hkv, n, d, gpu)
    win = ms.make_window(1, n, Hq, Hkv, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    grads = ms.window_bwd(win, q, k, v, out, do, lse)
    torch.cuda.synchronize()
    _check(q, k, v, do, out, lse, grads, W, S, d ** -0.5)


@pytest.mark.parametrize("B,n", [(1, 200), (64, 200)])
@pytest.mark.parametrize("W,S", [(1, 0), (4, 0), (20, 4), (60, 4)])
def test_window_few_keys_gradient_error(gpu, B, n, W, S):
    """Rows that see few keys: dQ and dK carry the roundings of dZ and of themselves to bf16, not that of O.  A rounding
    moves m 2^e (1 <= m < 2) by a uniformly spread error of at most 2^-8 2^e: 2^-8 / (m sqrt(3)) rms of the value, 0.736
    of 2^-8 / sqrt(3) over a binade of evenly spread logarithms, 1.66e-3; two of them are 2.35e-3 by the norms, and
    2.7e-3 leaves 15 %.  (With O's rounding: 3.0e-3 for 4 keys.)
    One key: P = 1 + t with |t| < 2^-20 (lse and its logit below 8 in log2 units, in fp32), dZ = -t dP with |dP| < 60,
    times scale |K| < 0.7: below 4e-5."""
    d, H = 64, 8
    q, k, v, do = _inputs(77, B, H, H, n, d, gpu)
    win = ms.make_window(B, n, H, H, d, W, S)
    out, lse = ms.window_fwd(win, q, k, v)
    dq, dk, _ = ms.window_bwd(win, q, k, v, out, do, lse)
    f = [to_f64(t[0].cpu()) for t in (q, k, v, do)]
    for got, (ref, _) in zip((dq, dk), OW.sequence_bwd(*f, W, S, d ** -0.5)):
        err = to_f64(got[0].cpu()) - ref
        if W == 1 and S == 0:
            assert np.abs(err).max() <= 4e-5
        else:
            assert np.linalg.norm(err) <= 2.7e-3 * np.linalg.norm(ref)


def test_window_far_strides(gpu):
    """Heads 2^31 elements apart: the same bits as in contiguous tensors."""
    n, d, gap = 150, 64, (1 << 31) + 64
    q, k, v, do = _inputs(81, 1, 2, 2, n, d, gpu)
    win = ms.make_window(1, n, 2, 2, d, 30, 2)
    out, lse = ms.window_fwd(win, q, k, v)
    want = (out, lse) + ms.window_bwd(win, q, k, v, out, do, lse)
    pool = torch.zeros(gap + 8 * n * d, dtype=torch.bfloat16, device=gpu)
    far = [pool.as_strided((1, 2, n, d), (0, gap, d, 1), i * n * d) for i in range(8)]
    for a, b in zip(far, (q, k, v, do)):
        a.copy_(b)
    fo, fl = ms.window_fwd(win, *far[:3], out=far[4])
    fg = ms.window_bwd(win, *far[:3], fo, far[3], fl, dq=far[5], dk=far[6], dv=far[7])
    for a, b in zip((fo, fl) + tuple(fg), want):
        assert torch.equal(a, b)


def test_window_two_calls_at_once(gpu):
    """Two streams, each with its own tensors and workspace; two graphs with one workspace, replayed in turn."""
    win = ms.make_window(1, 600, 4, 2, 64, 128, 70)
    data = [_inputs(90 + 10 * i, 1, 4, 2, 600, 64, gpu) for i in range(2)]

    def step(x, ws):
        out, lse = ms.window_fwd(win, *x[:3])
        return (out, lse) + ms.window_bwd(win, *x[:3], out, x[3], lse, workspace=ws)

    room = lambda: torch.empty(ms.window_bwd_workspace_bytes(win), dtype=torch.uint8, device=gpu)  # noqa: E731
    want = [step(x, room()) for x in data]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in data], []
    rooms = [room() for _ in data]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for s, x, ws in zip(streams, data, rooms):
            with torch.cuda.stream(s):
                got.append(step(x, ws))
    torch.cuda.synchronize()
    shared, graphs, outs = room(), [], []
    for x in data:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(x, shared))
        graphs.append(g)
    for _ in range(3):
        for g in graphs:   # one after the other on one stream
            g.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(got, want, outs):
            for x, y, z in zip(a, b, c):
                assert torch.equal(x, y) and torch.equal(z, y)


@pytest.mark.parametrize("lens,Hq,Hkv,d,W,S", [
    ([900, 0, 1700, 300], 4, 1, 128, 0, 0), ([2500, 40, 700], 2, 2, 64, 0, 0), ([1300, 1000], 14, 2, 128, 800, 4),
])
def test_window_packed_keys_in_several_walks(gpu, lens, Hq, Hkv, d, W, S):
    """Documents whose key groups' walks are cut for the mean one."""
    starts = torch.tensor([0] + lens).cumsum(0).to(torch.int32)
    total = int(starts[-1])
    q, k, v, do = _inputs(total, 1, Hq, Hkv, total, d, gpu)
    win = ms.make_window(len(lens), max(lens), Hq, Hkv, d, W, S, tokens=total)
    st = starts.to(gpu)
    out, lse = ms.window_fwd(win, q, k, v, starts=st)
    grads = ms.window_bwd(win, q, k, v, out, do, lse, starts=st)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        if n:
            _check(q, k, v, do, out, lse, grads, W, S, d ** -0.5, int(starts[b]), n)
