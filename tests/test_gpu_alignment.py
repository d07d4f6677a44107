"""int32 and fp32 arrays off their elements are refused by the calls around the output layer, before anything is launched."""
import ctypes

import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build

pytestmark = pytest.mark.gpu
ALIGNMENT = -2


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def refuses(ctx, fn, args, arrays):
    """``fn(ctx, *args)`` works, and is refused with any one of the arguments at ``arrays`` two bytes further on."""
    raw = [a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args]
    assert fn(ctx.h, *raw) == 0
    torch.cuda.synchronize()
    launches = ctx.launch_count()
    for i in arrays:
        moved = list(raw)
        moved[i] += 2
        assert fn(ctx.h, *moved) == ALIGNMENT, i
        assert b"aligned" in ctx.lib.jp_last_error(ctx.h)
    assert ctx.launch_count() == launches


def f32(*shape):
    return torch.rand((*shape, 2), device="cuda")[..., 0].contiguous() + 0.5


def test_norms(ctx):
    T, H = 6, 64
    x, dy, dx, w = f32(T, H), f32(T, H), f32(T, H), f32(H)
    mean, rstd, dw, db = f32(T), f32(T), f32(H), f32(H)
    ws = torch.empty(B.jp_layer_norm_workspace_bytes(ctx, T, H, B.JP_F32), dtype=torch.uint8, device="cuda")
    d = B.jp_norm_desc(T=T, H=H, dtype=B.JP_F32, param_dtype=B.JP_F32, eps=1e-6)
    refuses(ctx, ctx.lib.jp_layer_norm_forward, (ctypes.byref(d), x, w, None, dx, mean, rstd), (1, 2, 4, 5, 6))
    refuses(ctx, ctx.lib.jp_layer_norm_backward, (ctypes.byref(d), dy, x, w, mean, rstd, dx, dw, db, ws, ws.numel()), (1, 2, 3, 4, 5, 6, 7, 8))


def test_verification(ctx):
    n, N, V = 3, 2, 64
    i32 = lambda *s: torch.ones(s, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.jp_verify_workspace_bytes(ctx, n, N, V, B.JP_F32, True), dtype=torch.uint8, device="cuda")
    d = B.jp_verify_desc(B=n, V=V, N=N, dtype=B.JP_F32)
    refuses(ctx, ctx.lib.jp_verify_draft,
            (ctypes.byref(d), f32(n, N + 1, V), f32(n, N, V), i32(n, N), i32(n), f32(n), f32(n, N) / 2, f32(n) / 2, i32(n), i32(n, N + 1),
             f32(n, N), f32(n, N + 1), ws, ws.numel()), range(1, 12))
