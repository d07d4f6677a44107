"""The norms from two host threads at once, each with a context and a stream of its own: widths of one kernel that need different
amounts of shared memory.  The calls are made from C, one after the other without Python between them, so that the two threads are
often inside a call at the same time."""
import ctypes
import subprocess
import threading

import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu

LOOP = r"""
typedef int (*forward_fn)(void*, const void*, const void*, const void*, const void*, void*, float*, float*);
typedef int (*backward_fn)(void*, const void*, const void*, const void*, const void*, const float*, const float*, void*, float*,
                           float*, void*, unsigned long);
int forward_loop(forward_fn f, int n, void* ctx, const void* d, const void* x, const void* w, void* y) {
  for (int i = 0; i < n; ++i) { int st = f(ctx, d, x, w, 0, y, 0, 0); if (st) return st; }
  return 0;
}
int backward_loop(backward_fn f, int n, void* ctx, const void* d, const void* dy, const void* x, const void* w, const float* r,
                  void* dx, float* dw, void* ws, unsigned long bytes) {
  for (int i = 0; i < n; ++i) { int st = f(ctx, d, dy, x, w, 0, r, dx, dw, 0, ws, bytes); if (st) return st; }
  return 0;
}
"""


@pytest.fixture(scope="module")
def loops(tmp_path_factory):
    jp_build.build()
    d = tmp_path_factory.mktemp("loops")
    (d / "loops.c").write_text(LOOP)
    subprocess.run(["gcc", "-O2", "-shared", "-fPIC", "-o", str(d / "loops.so"), str(d / "loops.c")], check=True)
    return ctypes.CDLL(str(d / "loops.so"))


def ptr(t):
    return ctypes.c_void_p(t.data_ptr())


# (width, rows) of the larger and the smaller call of one kernel
@pytest.mark.parametrize("backward,dtype,large,small", [
    (False, torch.bfloat16, (16384, 4), (8200, 4)),           # a block a row: 98,304 and 55,296 bytes
    (False, torch.bfloat16, (4096, 1800), (2056, 1800)),      # a warp a row
    (True, torch.bfloat16, (8192, 4), (3000, 4)),
    (True, torch.float32, (8192, 4), (4500, 4)),
])
def test_two_threads_with_a_context_each(loops, backward, dtype, large, small):
    lib, n = B.load(), 20000 if large[1] < 100 else 2000
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [B.Context(0, s.cuda_stream) for s in streams]
    calls, outs, wants, keep = [], [], [], []
    for ctx, (H, T) in zip(ctxs, (large, small)):
        x, dy = (torch.randn((T, H), device="cuda").to(dtype) for _ in range(2))
        w, r = torch.rand(H, device="cuda") + 0.5, torch.rand(T, device="cuda") + 0.5
        d = B.jp_norm_desc(T=T, H=H, dtype=B._dtype_code(x), param_dtype=B.JP_F32, flags=B.JP_NORM_RMS, eps=1e-6)
        out = torch.zeros_like(x)
        if backward:
            wants.append(runner.layer_norm_backward(ctx, dy, x, w, None, r, rms=True, bias=False)[0])
            dw, ws = torch.empty(H, device="cuda"), torch.empty(B.jp_layer_norm_workspace_bytes(ctx, T, H, d.dtype), dtype=torch.uint8, device="cuda")
            calls.append((loops.backward_loop, lib.jp_layer_norm_backward, n, ctx.h, ctypes.byref(d), ptr(dy), ptr(x), ptr(w), ptr(r),
                          ptr(out), ptr(dw), ptr(ws), ctypes.c_ulong(ws.numel())))
            keep.append((dw, ws))
        else:
            wants.append(runner.layer_norm(ctx, x, w, eps=1e-6, rms=True)[0])
            calls.append((loops.forward_loop, lib.jp_layer_norm_forward, n, ctx.h, ctypes.byref(d), ptr(x), ptr(w), ptr(out)))
        outs.append(out)
        keep.append((x, dy, w, r, d))
    torch.cuda.synchronize()
    status, start = [None, None], threading.Barrier(2)

    def work(i):
        start.wait()
        status[i] = calls[i][0](*calls[i][1:])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert status == [0, 0], [c.lib.jp_last_error(c.h) for c in ctxs]
    assert all(torch.equal(o, w) for o, w in zip(outs, wants))
    for c in ctxs:
        c.close()
