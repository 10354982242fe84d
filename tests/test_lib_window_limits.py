"""Host-side limits of the window attention: what is refused before any launch, and what is accepted (by its workspace:
0 for a call that is refused)."""
import ctypes

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
