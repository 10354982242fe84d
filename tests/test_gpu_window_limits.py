"""Window attention on the largest grids.  Against the fp64 oracle as in test_gpu_window.py."""
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
