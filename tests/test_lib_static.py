"""Host-side checks of the static-pattern attention and the paged cache: refusals before any launch (fake pointers
that are never dereferenced), workspace queries, and the oracle's own pins."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_18830_amd as ms
from oracle import cache as OC
from oracle import window as OW

P16 = 4096
OK = dict(batch=2, seq=100, heads_q=4, heads_kv=2, head_dim=64, window=10, sinks=2)


def _tensor(h, n=100, d=64, data=P16, token=None, head=None, batch=None):
    token = d if token is None else token
    head = n * d if head is None else head
    return ms.Tensor(data, h * n * d if batch is None else batch, head, token)


def _fwd(win, starts=None, q=None, k=None, v=None, out=None, lse=P16):
    return ms.lib().msparse_window_fwd(win, starts, q or _tensor(4), k or _tensor(2), v or _tensor(2), out or _tensor(4),
                                       ctypes.c_void_p(lse), None)


def _message():
    return ms.lib().msparse_last_error().decode()


@pytest.mark.parametrize("change,status", [
    (dict(batch=0), -1), (dict(seq=-1), -1), (dict(heads_q=0), -1), (dict(heads_kv=3), -1), (dict(head_dim=96), -2),
    (dict(window=-1), -1), (dict(sinks=-1), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
    (dict(tokens=-1), -1), (dict(tokens=200), -1), (dict(seq=1 << 30), -2), (dict(batch=1 << 22, seq=1), -2),
])
def test_window_refuses_sizes(change, status):
    win = ms.make_window(**{**OK, **change})
    assert _fwd(win) == status, _message()
    assert ms.lib().msparse_window_bwd_workspace(win) == 0 or change == dict(tokens=200)


def test_window_refuses_tensors():
    win = ms.make_window(**OK)
    assert _fwd(win, q=_tensor(4, data=None)) == -1 and "NULL" in _message()
    assert _fwd(win, k=_tensor(2, data=P16 + 8)) == -1 and "16-byte" in _message()
    assert _fwd(win, v=_tensor(2, token=68)) == -1 and "stride" in _message()
    assert _fwd(win, v=_tensor(2, token=-64)) == -1
    assert _fwd(win, q=_tensor(4, head=1 << 62)) == -1
    assert _fwd(win, out=_tensor(4, token=0)) == -1 and "overlaps" in _message()
    assert _fwd(win, out=_tensor(4, head=64)) == -1 and "overlaps" in _message()
    assert _fwd(win, lse=None) == -1
    assert _fwd(win, lse=P16 + 4) == -1
    assert _fwd(win, starts=ctypes.c_void_p(P16)) == -1 and "starts" in _message()
    packed = ms.make_window(**{**OK, "tokens": 150})
    assert _fwd(packed) == -1 and "starts" in _message()
    assert _fwd(packed, starts=ctypes.c_void_p(P16 + 2)) == -1


def test_window_bwd_refuses():
    win = ms.make_window(**OK)
    need = ms.window_bwd_workspace_bytes(win)
    assert need > 0

    def call(ws=P16, room=need, dk=None, lse=P16):
        t = _tensor
        return ms.lib().msparse_window_bwd(win, None, t(4), t(2), t(2), t(4), t(4), ctypes.c_void_p(lse), t(4),
                                           dk or t(2), t(2), ctypes.c_void_p(ws), room, None)

    assert call(room=need - 1) == -4 and call(ws=None) == -4 and call(lse=None) == -1
    assert call(dk=_tensor(2, token=0)) == -1 and "dk" in _message()


def test_empty_calls_do_nothing():
    win = ms.make_window(**{**OK, "seq": 0})
    assert _fwd(win, q=_tensor(4, 0, data=None), out=_tensor(4, 0, data=None), lse=None) == 0
    c = _cache()
    assert ms.lib().msparse_cache_append(c, 4, 0, None, _tensor(2, 0), _tensor(2, 0), None, None, None, None) == 0
    assert ms.lib().msparse_cache_attn(c, 4, 0, 0, 0, 0.0, _tensor(4, 0), _tensor(4, 0), None, None, 0, None) == 0


def _cache(**change):
    f = dict(k=P16, v=P16, k_scale=P16, v_scale=P16, page_table=P16, lens=P16, pages=10, width=4, batch=2, heads_kv=2,
             head_dim=64)
    f.update(change)
    return ms.CacheStruct(*(f[n] for n, _ in ms.CacheStruct._fields_))


CACHE_REFUSALS = [
    (dict(batch=0), -1), (dict(heads_kv=0), -1), (dict(heads_kv=3), -1), (dict(head_dim=80), -2), (dict(pages=0), -1),
    (dict(width=0), -1), (dict(width=(1 << 24) + 1), -2), (dict(k=None), -1), (dict(v=P16 + 8), -1),
    (dict(k_scale=None), -1), (dict(v_scale=P16 + 2), -1), (dict(page_table=None), -1), (dict(lens=None), -1),
]


@pytest.mark.parametrize("change,status", CACHE_REFUSALS)
def test_cache_refuses(change, status):
    c, t = _cache(**change), _tensor
    n = 5
    L = ms.lib()
    kv = t(2, n)
    assert L.msparse_cache_append(c, 4, n, t(4, n), kv, kv, t(4, n), None, None, None) == status, _message()
    assert L.msparse_cache_attn(c, 4, n, 0, 0, 0.0, t(4, n), t(4, n), None, ctypes.c_void_p(P16), 1 << 40,
                                None) == status, _message()


def test_cache_refuses_arguments():
    c, t, n, L = _cache(), _tensor, 5, ms.lib()
    kv = t(2, n)

    def append(tokens=n, q=t(4, n), k=kv, qo=t(4, n, data=2 * P16), freq=None, counts=None):
        return L.msparse_cache_append(c, 4, tokens, q, k, kv, qo, freq, counts, None)

    assert append(tokens=-1) == -1 and append(q=None) == -1 and append(qo=None) == -1
    assert append(k=None) == -1 and append(k=t(2, n, token=4)) == -1
    assert append(qo=t(4, n, token=0)) == -1
    assert append(freq=ctypes.c_void_p(P16 + 1)) == -1 and append(counts=ctypes.c_void_p(P16 + 2)) == -1
    assert append(qo=t(4, n, token=128, head=128 * n, batch=4 * 128 * n, data=P16)) == -1 and "in place" in _message()
    assert append(tokens=1 << 30) == -2

    def attn(window=0, sinks=0, scale=0.0, q=t(4, n), out=t(4, n), ws=P16, room=1 << 40):
        return L.msparse_cache_attn(big, 4, n, window, sinks, scale, q, out, None, ctypes.c_void_p(ws), room, None)

    big = _cache(width=1000)
    need = L.msparse_cache_attn_workspace(big, 4, n)
    assert need > 0 and L.msparse_cache_attn_workspace(_cache(width=4), 4, n) == 0
    assert attn(window=-1) == -1 and attn(sinks=-1) == -1 and attn(scale=float("nan")) == -1
    assert attn(q=None) == -1 and attn(out=t(4, n, head=0)) == -1
    assert attn(room=need - 1) == -4 and attn(ws=None) == -4 and attn(ws=P16 + 4) == -1


def test_binding_refuses_host_tensors_and_types():
    q = torch.zeros((1, 2, 8, 64), dtype=torch.bfloat16)
    win = ms.make_window(1, 8, 2, 2, 64)
    with pytest.raises(ms.MsparseError):
        ms.window_fwd(win, q, q, q)
    cache = ms.make_cache(2, 2, 64, "cpu")
    table = torch.zeros((1, 1), dtype=torch.int32)
    lens = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ms.MsparseError):
        ms.cache_append(cache, table, lens, q, q)
    with pytest.raises(ms.MsparseError):
        ms.cache_attn(cache, table, lens, q)


# ---------------------------------------------------------------- the oracle's pins
def test_oracle_window_mask_by_loops():
    for n, W, S in ((9, 3, 2), (7, 0, 3), (5, 1, 0), (6, 2, 6), (1, 1, 1)):
        m = OW.mask(n, W, S)
        for i in range(n):
            for j in range(n):
                assert m[i, j] == (j <= i and (W == 0 or i - j < W or j < S))


def test_oracle_window_against_autograd():
    rng = np.random.default_rng(0)
    q, k, v, do = (rng.standard_normal((h, 23, 8)) for h in (4, 2, 2, 4))
    t = [torch.from_numpy(x).requires_grad_() for x in (q, k, v)]
    z = (t[0].view(2, 2, 23, 8) @ t[1].view(2, 1, 23, 8).transpose(-1, -2)) * 0.4
    z = z.masked_fill(~torch.from_numpy(OW.mask(23, 6, 2)), -np.inf)
    o = (torch.softmax(z, -1) @ t[2].view(2, 1, 23, 8)).view(4, 23, 8)
    (o * torch.from_numpy(do)).sum().backward()
    out, _, lse, _ = OW.sequence_fwd(q, k, v, 6, 2, 0.4)
    assert np.allclose(out, o.detach().numpy(), atol=1e-12)
    assert np.allclose(lse, torch.logsumexp(z, -1).view(4, 23).detach().numpy(), atol=1e-12)
    for got, x in zip(OW.sequence_bwd(q, k, v, do, 6, 2, 0.4), t):
        assert np.allclose(got[0], x.grad.numpy(), atol=1e-12)


def test_oracle_e4m3_against_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(OC.DECODE, want, equal_nan=True)
    x = np.random.default_rng(1).standard_normal(20000).astype(np.float32) * 60
    x = np.concatenate([x, 2.0 ** -np.arange(1, 14), want[:127], (want[:126] + want[1:127]) / 2]).astype(np.float32)
    x = np.concatenate([x, -x])
    x = x[np.abs(x) <= 448]
    got = OC.encode(x)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(got, ref)


def test_oracle_scale_is_the_smallest_power_of_two():
    for amax in (1e-45, 1.0, 447.9, 448.0, 448.1, 14.0, 14.01, 3.3e38):
        s = OC.scale_of(amax)
        assert amax <= 448 * s and (s == 2.0 ** -126 or amax > 224 * s)
    assert OC.scale_of(0.0) == 2.0 ** -126


def test_oracle_append_in_parts_keeps_the_values():
    """Tokens appended one by one hold, within one code's rounding twice, the values that they came with."""
    rng = np.random.default_rng(2)
    d, n = 8, 70
    x, y = rng.standard_normal((1, 1, n, d)), rng.standard_normal((1, 1, n, d))
    table = np.array([[1, 0]])
    k, v = np.zeros((2, 1, 64, d), np.uint8), np.zeros((2, 1, d, 64), np.uint8)
    ks, vs = np.ones((2, 1)), np.ones((2, 1))
    for t in range(n):
        OC.append(k, v, ks, vs, table, [t], x[:, :, t:t + 1], y[:, :, t:t + 1], [1], None)
    kk, vv, have = OC.gather(k, v, ks, vs, table, n, 0, 0)
    assert have.all()
    for got, want in ((kk, x[0, 0]), (vv, y[0, 0])):
        assert (np.abs(got - want) <= 2.0 ** -3 * np.abs(want) + 2.0 ** -9).all()
