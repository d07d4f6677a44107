"""Calls that need more shared memory than every kernel has, before and after the process resets its own context on the device (a child process: torch's
context would go with it)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import ctypes
from cuda.bindings import driver
from paper_2602_06107_b200 import binding as B

def answer(r):
    assert r[0] == driver.CUresult.CUDA_SUCCESS, r[0]
    return r[1] if len(r) > 1 else None

def calls():
    lib, h = B.load(), ctypes.c_void_p()
    assert lib.jp_create(ctypes.byref(h), 0, None) == 0
    mem, MB = int(answer(driver.cuMemAlloc(64 << 20))), 1 << 20
    answer(driver.cuMemsetD8(mem, 0, 64 << 20))
    loss = B.jp_policy_desc(T=4, V=200000, dtype=B.JP_BF16, eps_lo=0.2, eps_hi=0.2)
    print(lib.jp_policy_loss(h, ctypes.byref(loss), mem + 32 * MB, mem, None, mem + MB, mem + MB, None, None, mem + 2 * MB, None, None, None, mem + 40 * MB,
                             mem + 3 * MB, lib.jp_policy_workspace_bytes(h, 4)))
    norm = B.jp_block_norm_desc(T=4, H=16384, dtype=B.JP_BF16, param_dtype=B.JP_F32, flags=B.JP_NORM_RMS, eps=1e-6, scale=1.0)
    print(lib.jp_block_norm_forward(h, ctypes.byref(norm), mem, mem, mem + MB, *[None] * 5, mem + 4 * MB, mem + 8 * MB, *[None] * 4))
    answer(driver.cuCtxSynchronize())
    lib.jp_destroy(h)

answer(driver.cuInit(0))
device = answer(driver.cuDeviceGet(0))
for turn in range(2):
    answer(driver.cuCtxSetCurrent(answer(driver.cuDevicePrimaryCtxRetain(device))))
    calls()
    answer(driver.cuDevicePrimaryCtxReset(device))
"""


@pytest.mark.gpu
def test_calls_after_the_context_was_reset():
    from paper_2602_06107_b200 import build as jp_build
    jp_build.build()
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert r.stdout.split() == ["0"] * 4
