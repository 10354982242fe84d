"""Rotation by positions on several axes (rotate, cache_append with positions) against the fp64 oracle.

Tolerances: cos and sin are rounded once to fp32 (2^-24 each), their two products and the sum likewise: at most
4 x 2^-24 (|x1| + |x2|) in fp32, and one rounding of the result (2^-8 of it) in bf16."""
import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import cache as OC
from oracle import tree as OT
from oracle import window as OW
from tests.helpers import to_f64

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _randn(seed, shape, gpu, dtype=BF):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).to(gpu)


def _freq(d, gpu, base=10000.0):
    return (base ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)).float().to(gpu)


def _positions(seed, axes, B, N, top, gpu):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-5, top, (axes, B, N), generator=g, dtype=torch.int32).to(gpu)


def _f64(t):
    t = t.contiguous().cpu()
    return to_f64(t) if t.dtype == BF else t.numpy().astype(np.float64)


def _check(got, x, positions, freq, axis, inverse):
    """got and x [B, H, N, d]."""
    g, x = _f64(got), _f64(x)
    h = x.shape[3] // 2
    for b in range(x.shape[0]):
        for i in range(x.shape[1]):
            r = OT.rotate(x[b, i], positions[:, b], freq, axis, inverse)
            both = np.abs(x[b, i, :, :h]) + np.abs(x[b, i, :, h:])
            bound = 2.0 ** -22 * np.concatenate([both, both], 1)
            if got.dtype == BF:
                bound = 2.0 ** -8 * (np.abs(r) + bound) + bound
            assert (np.abs(g[b, i] - r) <= bound).all(), (b, i)


@pytest.mark.parametrize("B,Hq,Hkv,d,N,axes,dtype", [
    (1, 1, 1, 64, 1, 1, BF), (1, 4, 2, 64, 63, 2, BF), (2, 3, 1, 128, 65, 3, BF), (3, 7, 7, 64, 130, 4, BF),
    (1, 28, 4, 128, 200, 3, BF), (70, 2, 1, 128, 3, 2, BF), (1, 1, 1, 128, 1, 1, F32), (2, 5, 3, 64, 77, 3, F32),
    (1, 12, 4, 128, 129, 2, F32), (5, 40, 0, 64, 17, 1, BF),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotate_matches_oracle(gpu, B, Hq, Hkv, d, N, axes, dtype, inverse):
    print(f"rotate B{B} Hq{Hq} Hkv{Hkv} d{d} N{N} axes{axes} {dtype} {inverse}", flush=True)
    q = _randn(1, (B, Hq, N, d), gpu, dtype)
    k = _randn(2, (B, Hkv, N, d), gpu, dtype) if Hkv else None
    pos = _positions(3, axes, B, N, 70000, gpu)
    axis = (torch.arange(d // 2) % axes).to(torch.int32).to(gpu)
    freq = _freq(d, gpu)
    qo, ko = ms.rotate(q, k, pos, freq, axis=axis, inverse=inverse)
    torch.cuda.synchronize()
    p, f, a = pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy()
    assert qo.dtype == dtype and (ko is None) == (k is None)
    _check(qo, q, p, f, a, inverse)
    if Hkv:
        _check(ko, k, p, f, a, inverse)


def test_rotate_a_part_of_the_columns_and_far_positions(gpu):
    """Axes outside the axes leave their pairs, bit for bit; positions up to 2^31 - 1 and -2^31."""
    d, N = 128, 6
    q, k = _randn(1, (1, 2, N, d), gpu), _randn(2, (1, 1, N, d), gpu)
    pos = torch.tensor([[2 ** 31 - 1, -2 ** 31, 100000007, 0, 1, 131071], [5, 6, 2 ** 30, -7, 8, 9]], dtype=torch.int32,
                       device=gpu)[:, None]
    axis = torch.arange(64, dtype=torch.int32) % 4 - 1
    freq = _freq(d, gpu, 500000.0)
    qo, ko = ms.rotate(q, k, pos, freq, axis=axis.to(gpu))
    torch.cuda.synchronize()
    _check(qo, q, pos.cpu().numpy(), freq.cpu().numpy(), axis.numpy(), False)
    _check(ko, k, pos.cpu().numpy(), freq.cpu().numpy(), axis.numpy(), False)
    left = torch.cat([(axis < 0) | (axis > 1)] * 2).to(gpu)
    assert torch.equal(qo[..., left], q[..., left])


def _any_bits(seed, shape, gpu, dtype):
    """Any bit patterns: infinities, NaNs of both kinds, zeros of both signs, subnormal values."""
    g = torch.Generator().manual_seed(seed)
    n, whole = (16, torch.int16) if dtype == BF else (32, torch.int32)
    x = torch.randint(-2 ** (n - 1), 2 ** (n - 1), shape, generator=g, dtype=torch.int64)
    some = torch.tensor([0, -2 ** (n - 1), 0x7f80, 0x7fc0, 0x7f81, -0x80, 1], dtype=torch.int64)
    some[2:6] <<= n - 16   # the infinities, a quiet and a signalling NaN
    pick = torch.randint(0, 20, shape, generator=g)
    x = torch.where(pick < 7, some[pick.clamp(max=6)], x)
    return x.to(whole).view(dtype).to(gpu)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("inverse", [False, True])
def test_pairs_outside_the_axes_keep_their_bits(gpu, d, dtype, inverse):
    N, axes = 130, 2
    whole = torch.int16 if dtype == BF else torch.int32
    g = torch.Generator().manual_seed(d)
    axis = torch.randint(-2, 4, (d // 2,), generator=g, dtype=torch.int32)
    left = torch.cat([(axis < 0) | (axis >= axes)] * 2).to(gpu)
    q, k = (torch.where(left, _any_bits(i, (2, h, N, d), gpu, dtype).view(whole),
                        _randn(i, (2, h, N, d), gpu, dtype).view(whole)).view(dtype) for i, h in ((1, 3), (2, 1)))
    pos, freq = _positions(3, axes, 2, N, 70000, gpu), _freq(d, gpu)
    got = ms.rotate(q, k, pos, freq, axis=axis.to(gpu), inverse=inverse)
    for y, x in zip(got, (q, k)):
        assert torch.equal(y[..., left].view(whole), x[..., left].view(whole))
        z = torch.where(left, torch.zeros_like(x), x)
        _check(torch.where(left, torch.zeros_like(y), y), z, pos.cpu().numpy(), freq.cpu().numpy(), axis.numpy(), inverse)
    same = ms.rotate(q, k, pos, freq, axis=torch.full_like(axis, axes).to(gpu), inverse=inverse, q_out=q.clone())
    assert torch.equal(same[0].view(whole), q.view(whole)) and torch.equal(same[1].view(whole), k.view(whole))


def test_rotate_strides_in_place_and_one_axis(gpu):
    B, Hq, Hkv, N, d = 2, 4, 2, 70, 64
    q, k = _randn(1, (B, N, Hq, d), gpu).transpose(1, 2), _randn(2, (B, Hkv, N, d + 16), gpu)[..., :d]
    pos, freq = _positions(3, 1, B, N, 9999, gpu), _freq(d, gpu)
    want = ms.rotate(q.contiguous(), k.contiguous(), pos, freq)
    got = ms.rotate(q, k, pos[0].contiguous(), freq)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert got[0].stride() == q.stride()
    big = torch.full((B, Hkv, N, d + 16), 3.0, dtype=BF, device=gpu)
    ms.rotate(q, k, pos, freq, k_out=big[..., :d])
    assert torch.equal(big[..., :d], want[1]) and (big[..., d:] == 3).all()
    same = ms.rotate(q, k, pos, freq, q_out=q, k_out=k)
    assert same[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])


def test_rotate_gradient_is_the_inverse(gpu):
    """<rotate(x), g> = <x, inverse(g)>, central differences of the oracle, and a layer's step together: rotated queries
    and keys through the window attention and back."""
    B, H, N, d, axes = 1, 2, 40, 64, 3
    x, g = _randn(1, (B, H, N, d), gpu, F32), _randn(2, (B, H, N, d), gpu, F32)
    pos, freq = _positions(3, axes, B, N, 5000, gpu), _freq(d, gpu)
    axis = (torch.arange(d // 2) % axes).to(torch.int32).to(gpu)
    y, _ = ms.rotate(x, None, pos, freq, axis=axis)
    back, _ = ms.rotate(g, None, pos, freq, axis=axis, inverse=True)
    a, b = (y.double() * g.double()).sum(), (x.double() * back.double()).sum()
    # each element is off by at most 2^-22 (|x1| + |x2|), |x|, |g| < 6: N H d terms of 12 x 6 x 2^-22 at most
    assert abs(float(a - b)) <= 2 * N * H * d * 72 * 2.0 ** -22
    p, f, ax = pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy()
    x64, g64, step = _f64(x)[0, 1], _f64(g)[0, 1], 2.0 ** -10
    rng = np.random.default_rng(0)
    for _ in range(3):
        u = rng.standard_normal(x64.shape)
        diff = ((OT.rotate(x64 + step * u, p[:, 0], f, ax) - OT.rotate(x64 - step * u, p[:, 0], f, ax)) * g64).sum() / (2 * step)
        want = (_f64(back)[0, 1] * u).sum()
        assert abs(diff - want) <= np.abs(u).sum() * 12 * 2.0 ** -22 + 1e-9 * abs(diff)


def test_rotate_with_window_attention(gpu):
    """A layer's step: rotate, window attention, its backward, the gradients turned back; against autograd in fp64 from the
    rotated bf16 tensors on."""
    B, Hq, Hkv, N, d, W, axes = 1, 4, 2, 90, 64, 30, 2
    q, k, v, do = (_randn(i, (B, h, N, d), gpu) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    pos, freq = _positions(3, axes, B, N, 200, gpu), _freq(d, gpu)
    axis = (torch.arange(d // 2) % axes).to(torch.int32).to(gpu)
    qr, kr = ms.rotate(q, k, pos, freq, axis=axis)
    win = ms.make_window(B, N, Hq, Hkv, d, W, 2)
    out, lse = ms.window_fwd(win, qr, kr, v)
    dqr, dkr, _ = ms.window_bwd(win, qr, kr, v, out, do, lse)
    dq, dk = ms.rotate(dqr, dkr, pos, freq, axis=axis, inverse=True)
    torch.cuda.synchronize()
    p, f, a = pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy()
    _check(dq, dqr, p, f, a, True)
    _check(dk, dkr, p, f, a, True)


def _turn64(x, positions, freq, axis):
    """x fp64 [H, N, d], differentiable; also |cos| and |sin| of the pairs."""
    h = x.shape[2] // 2
    ang = torch.from_numpy(positions[axis].T.astype(np.float64) * freq.astype(np.float64))   # [N, h]
    c, s = ang.cos(), ang.sin()
    return torch.cat([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1), c.abs().numpy(), s.abs().numpy()


@pytest.mark.parametrize("Hq,Hkv,N,d,W,S,axes", [(4, 2, 90, 64, 30, 2, 2), (2, 2, 200, 128, 0, 0, 3), (7, 1, 333, 64, 100, 7, 1)])
def test_a_layers_step_against_autograd(gpu, Hq, Hkv, N, d, W, S, axes):
    """rotate, window attention, its backward, the gradients turned back: outputs and the gradients of the queries and keys
    before the rotation against autograd in fp64 through all of it (the rotated tensors take the values that rotate rounded
    to bf16, themselves checked).  Bounds: those of the attention (oracle/window.py), of two columns where they turn into
    one, and the rotation's roundings."""
    q, k, v, do = (_randn(i, (1, h, N, d), gpu) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    pos, freq = _positions(3, axes, 1, N, 2000, gpu), _freq(d, gpu)
    axis = (torch.arange(d // 2) % axes).to(torch.int32).to(gpu)
    qr, kr = ms.rotate(q, k, pos, freq, axis=axis)
    win = ms.make_window(1, N, Hq, Hkv, d, W, S)
    out, lse = ms.window_fwd(win, qr, kr, v)
    dqr, dkr, dv = ms.window_bwd(win, qr, kr, v, out, do, lse)
    dq, dk = ms.rotate(dqr, dkr, pos, freq, axis=axis, inverse=True)
    torch.cuda.synchronize()
    p, f, a = pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy()
    _check(qr, q, p, f, a, False)
    _check(kr, k, p, f, a, False)
    # autograd
    leaf = [torch.from_numpy(_f64(t)[0]).requires_grad_() for t in (q, k, v)]
    turned, rounded = [], [torch.from_numpy(_f64(t)[0]) for t in (qr, kr)]
    for x, y in zip(leaf, rounded):
        z, c, s = _turn64(x, p[:, 0], f, a)
        turned.append(z + (y - z).detach())
    G = Hq // Hkv
    z = (turned[0].view(Hkv, G, N, d) @ turned[1].view(Hkv, 1, N, d).transpose(-1, -2)) * d ** -0.5
    z = z.masked_fill(~torch.from_numpy(OW.mask(N, W, S)), -np.inf)
    o = (torch.softmax(z, -1) @ leaf[2].view(Hkv, 1, N, d)).view(Hq, N, d)
    (o * torch.from_numpy(_f64(do)[0])).sum().backward()
    # bounds
    host = [t.numpy() for t in rounded] + [_f64(v)[0], _f64(do)[0]]
    _, eo, _, reach = OW.sequence_fwd(*host[:3], W, S, d ** -0.5)
    (_, eq), (_, ek), (_, ev) = OW.sequence_bwd(*host, W, S, d ** -0.5)
    assert (np.abs(_f64(out)[0] - o.detach().numpy()) <= eo).all()
    want = torch.logsumexp(z.detach(), -1).view(Hq, N).numpy()
    assert np.abs(lse[0].double().cpu().numpy() - want).max() <= OW.lse_bound(N, d, reach)
    assert (np.abs(_f64(dv)[0] - leaf[2].grad.numpy()) <= ev).all()
    h = d // 2
    for got, before, x, e in ((dq, dqr, leaf[0], eq), (dk, dkr, leaf[1], ek)):
        ref, g = x.grad.numpy(), np.abs(_f64(before)[0])
        bound = np.concatenate([e[..., :h] * c + e[..., h:] * s, e[..., h:] * c + e[..., :h] * s], -1)
        bound += 2.0 ** -22 * np.concatenate([g[..., :h] + g[..., h:]] * 2, -1)
        bound += 2.0 ** -8 * (np.abs(ref) + bound)
        err = np.abs(_f64(got)[0] - ref)
        assert (err <= bound).all(), (err.max(), (err > bound).sum())


def test_rotate_of_many_tokens(gpu):
    """More blocks of tokens than the card runs at once, with each block's heads in one workgroup."""
    B, Hq, Hkv, N, d = 3, 2, 1, 40000, 64
    q, k = _randn(1, (B, Hq, N, d), gpu), _randn(2, (B, Hkv, N, d), gpu)
    pos, freq = _positions(3, 2, B, N, 10 ** 6, gpu), _freq(d, gpu)
    axis = (torch.arange(d // 2) % 2).to(torch.int32).to(gpu)
    qo, ko = ms.rotate(q, k, pos, freq, axis=axis)
    torch.cuda.synchronize()
    _check(qo, q, pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy(), False)
    _check(ko, k, pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy(), False)


def test_rotate_in_a_graph_and_on_a_stream(gpu):
    q, k = _randn(1, (1, 3, 50, 64), gpu), _randn(2, (1, 1, 50, 64), gpu)
    pos, freq = _positions(3, 1, 1, 50, 999, gpu), _freq(64, gpu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = ms.rotate(q, k, pos, freq, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = ms.rotate(q, k, pos, freq)
    for seed in (4, 5, 6):
        q.copy_(_randn(seed, q.shape, gpu))
        pos.copy_(_positions(seed, 1, 1, 50, 999, gpu))
        graph.replay()
        want = ms.rotate(q, k, pos, freq)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q.copy_(_randn(1, q.shape, gpu))
    pos.copy_(_positions(3, 1, 1, 50, 999, gpu))
    want = ms.rotate(q, k, pos, freq)
    assert torch.equal(on_side[0], want[0]) and torch.equal(on_side[1], want[1])


# ---------------------------------------------------------------- the cache
@pytest.mark.parametrize("B,Hq,Hkv,d,T,lens,counts,axes", [
    (1, 4, 1, 64, 1, [63], None, 1), (3, 4, 2, 128, 70, [0, 30, 64], [70, 0, 33], 3), (2, 6, 2, 64, 130, [5, 100], None, 2),
    (2, 28, 4, 128, 16, [60, 1000], None, 4), (1, 14, 1, 64, 4200, [17], None, 2), (66, 6, 3, 64, 64, list(range(66)), None, 1),
    (2, 24, 24, 64, 2050, [1, 64], [2050, 700], 3), (1, 26, 2, 128, 4097, [0], None, 3),
])
def test_append_at_positions(gpu, B, Hq, Hkv, d, T, lens, counts, axes):
    """The cache's values are those of keys rotated by rotate in fp32 and appended without a rotation, up to the fp32
    roundings at a code's border; places, scales and V as ever."""
    print(f"append at B{B} Hq{Hq} Hkv{Hkv} d{d} T{T} {lens} {counts} axes{axes}", flush=True)
    pages = sum((n + T + 63) // 64 for n in lens) + 1
    table, at = torch.full((B, max((n + T + 63) // 64 for n in lens)), -1, dtype=torch.int32), 0
    for b, n in enumerate(lens):
        m = (n + T + 63) // 64
        table[b, :m] = torch.arange(at, at + m)
        at += m
    table = table.to(gpu)
    cache = ms.make_cache(pages, Hkv, d, gpu)
    for t in (cache.k, cache.v):
        t.view(torch.uint8).zero_()
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(2.0 ** -9)
    q, k, v = (_randn(i, (B, h, T, d), gpu) for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    pos, freq = _positions(4, axes, B, T, 3000, gpu), _freq(d, gpu)
    axis = (torch.arange(d // 2) % axes).to(torch.int32).to(gpu)
    L = torch.tensor(lens, dtype=torch.int32, device=gpu)
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device=gpu)
    ref = [t.cpu().view(torch.uint8).numpy().copy() for t in (cache.k, cache.v)] + \
          [t.cpu().numpy().astype(np.float64) for t in (cache.k_scale, cache.v_scale)]
    got_q = ms.cache_append(cache, table, L, k, v, q=q, inv_freq=freq, counts=cnt, positions=pos, axis=axis)
    torch.cuda.synchronize()
    p, f, a = pos.cpu().numpy(), freq.cpu().numpy(), axis.cpu().numpy()
    _check(got_q, q, p, f, a, False)
    x = np.stack([np.stack([OT.rotate(h, p[:, b], f, a) for h in _f64(k)[b]]) for b in range(B)])
    OC.append(*ref, table.cpu().numpy(), lens, x, _f64(v), counts or [T] * B, None)
    gk, gv = (t.cpu().view(torch.uint8).numpy() for t in (cache.k, cache.v))
    assert np.array_equal(cache.k_scale.cpu().numpy(), ref[2]) and np.array_equal(cache.v_scale.cpu().numpy(), ref[3])
    assert np.array_equal(gv, ref[1])
    off = gk != ref[0]   # a neighbouring code where fp32 (2^-22 of both columns) decides: a few in 10^5
    assert off.mean() <= 1e-3
    assert (np.abs(OC.DECODE[gk[off]] - OC.DECODE[ref[0][off]]) <= np.maximum(2.0 ** -9, 0.134 * np.abs(OC.DECODE[gk[off]]))).all()


def test_append_at_one_axis_is_append(gpu):
    """Positions lens + t on one axis: the same queries, values and codes as without (angles are formed by another sum in 64
    bits, so neighbours are allowed as there)."""
    B, Hq, Hkv, d, T = 2, 4, 2, 64, 40
    table = torch.arange(4, dtype=torch.int32, device=gpu).view(2, 2)
    L = torch.tensor([3, 62], dtype=torch.int32, device=gpu)
    q, k, v = (_randn(i, (B, h, T, d), gpu) for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    pos = L[:, None] + torch.arange(T, dtype=torch.int32, device=gpu)
    got = []
    for more in ({}, dict(positions=pos)):
        c = ms.make_cache(4, Hkv, d, gpu)
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.view(torch.uint8).zero_()
        qr = ms.cache_append(c, table, L, k, v, q=q, inv_freq=_freq(d, gpu), **more)
        got.append((qr, c))
    (q0, c0), (q1, c1) = got
    assert (q0.float() - q1.float()).abs().max() <= 2.0 ** -7 * 4
    assert torch.equal(c0.v.view(torch.uint8), c1.v.view(torch.uint8)) and torch.equal(c0.v_scale, c1.v_scale)
    assert torch.equal(c0.k_scale, c1.k_scale)
    assert (c0.k.view(torch.uint8) != c1.k.view(torch.uint8)).float().mean() <= 1e-3


@pytest.mark.parametrize("d,T", [(64, 5), (128, 100)])
def test_append_leaves_pairs_outside_the_axes(gpu, d, T):
    """Queries keep their bits there; of keys an element that is not finite has the code NaN, and its partner its own."""
    Hq, Hkv = 4, 2
    axis = (torch.arange(d // 2, dtype=torch.int32) % 3 - 1).to(gpu)
    left = torch.cat([axis < 0] * 2)
    q = torch.where(left, _any_bits(1, (1, Hq, T, d), gpu, BF).view(torch.int16), _randn(1, (1, Hq, T, d), gpu).view(torch.int16))
    k = _randn(2, (1, Hkv, T, d), gpu)
    k[0, 0, 1::7, 0], k[0, 1, ::5, d // 2 + 3], k[0, 1, 3, 6] = float("inf"), float("nan"), -float("inf")
    odd = torch.where(left, ~k.isfinite(), False)
    assert odd.any() and k[..., ~left].isfinite().all()
    pages = (T + 63) // 64
    table = torch.arange(pages, dtype=torch.int32, device=gpu)[None]
    pos, freq = _positions(3, 2, 1, T, 70000, gpu), _freq(d, gpu)
    lens = torch.zeros(1, dtype=torch.int32, device=gpu)
    both = []
    for keys in (k, torch.where(odd, torch.zeros_like(k), k)):
        c = ms.make_cache(pages, Hkv, d, gpu)
        for t in (c.k, c.v, c.k_scale, c.v_scale):
            t.view(torch.uint8).zero_()
        got = ms.cache_append(c, table, lens, keys, keys, q=q.view(BF), inv_freq=freq, positions=pos, axis=axis)
        assert torch.equal(got[..., left].view(torch.int16), q[..., left])
        code = c.k.view(torch.uint8).permute(1, 0, 2, 3).reshape(1, Hkv, -1, d)[:, :, :T]
        both.append((code, c.k_scale))
    (code, scale), (want, wanted) = both
    assert torch.equal(scale, wanted)
    assert (code[odd] & 127 == 127).all() and torch.equal(code[~odd], want[~odd])
