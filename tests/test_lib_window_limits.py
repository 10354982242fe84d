"""Host-side limits of the window attention: what is refused before any launch, and what is accepted (by its workspace:
0 for a call that is refused)."""
import ctypes

import pytest

import paper_2510_18830_amd as ms

P16 = 4096


def _bwd(win):
    n, d = win.seq, win.head_dim
    t = lambda h: ms.Tensor(P16, h * n * d, n * d, d)  # noqa: E731
    q, k = t(win.heads_q), t(win.heads_kv)
    return ms.lib().msparse_window_bwd(win, None, q, k, k, q, q, ctypes.c_void_p(P16), q, k, k, ctypes.c_void_p(P16),
                                       1 << 62, None)


def test_window_bwd_refuses_a_launch_of_2_to_the_32_threads():
    """2^22 groups of keys, which the forward takes, and as many chunks of their sinks, of 512 threads each."""
    win = ms.make_window(1 << 22, 64, 1, 1, 128, 1, 1)
    assert _bwd(win) == -2 and "2^23" in ms.lib().msparse_last_error().decode()
    assert ms.window_bwd_workspace_bytes(win) == 0
    assert ms.window_bwd_workspace_bytes(ms.make_window(1 << 21, 64, 1, 1, 128, 1, 1)) > 0


def test_window_packed_is_limited_by_its_rows():
    """Many documents of which one may be long, or whose longest the caller does not know: the tensors' rows count, not
    documents times the longest."""
    for docs, tokens, longest, heads_q, heads_kv, d in ((80, 1 << 19, 1 << 17, 28, 4, 128), (128, 1 << 18, 1 << 17, 32, 8, 64),
                                                        (200, 1 << 17, 1 << 16, 32, 8, 128), (100, 131072, 131072, 32, 8, 128),
                                                        (300, 300 * 500, 1 << 15, 32, 32, 64), (5000, 131072, 131072, 16, 2, 128)):
        for W, S in ((0, 0), (4096, 0), (512, 4)):
            win = ms.make_window(docs, longest, heads_q, heads_kv, d, W, S, tokens=tokens)
            need = ms.window_bwd_workspace_bytes(win)
            rows = 8 * heads_q * (tokens + 64 * docs)   # lse and Delta of a row
            groups = heads_kv * (docs + tokens // 512)  # ones that may have rows beyond the window, and their chunks
            assert rows <= need <= 1.02 * rows + (3 * groups + 2048 * heads_kv) * 2 * 128 * d * 4 * (S > 0)
    win = ms.make_window(1 << 21, 1 << 20, 8, 8, 64, 100, 4, tokens=1 << 20)
    assert ms.window_bwd_workspace_bytes(win) == 0 and "blocks of 64 rows" in ms.lib().msparse_last_error().decode()


@pytest.mark.parametrize("W,S", [(0, 0), (100, 4), (100, 290)])
def test_window_packed_longest_beyond_the_rows(W, S):
    """No document is longer than the tensors: `seq` beyond them plans what `tokens` plans."""
    need = [ms.window_bwd_workspace_bytes(ms.make_window(3, seq, 128, 1, 64, W, S, tokens=300)) for seq in (300, 301, 1 << 30)]
    assert need[0] == need[1] == need[2] > 0
