"""The structs of the calls around the output layer as gcc sees them in the header against their ctypes mirrors, and what those
calls answer without a context (no device is needed)."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"jp_norm_desc": B.jp_norm_desc, "jp_w4_desc": B.jp_w4_desc, "jp_verify_desc": B.jp_verify_desc}


def test_structs_match_the_header(tmp_path):
    prints = "".join(f'printf("%zu ", sizeof({n}));' + "".join(f'printf("%zu ", offsetof({n}, {f}));' for f, _ in c._fields_)
                     for n, c in STRUCTS.items())
    src = tmp_path / "sz.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "jackpot.h"\nint main(void){' + prints + 'return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for c in STRUCTS.values():
        want += [ctypes.sizeof(c)] + [getattr(c, f).offset for f, _ in c._fields_]
    assert got == want


def test_limits_match_the_header(tmp_path):
    src = tmp_path / "lim.c"
    src.write_text('#include <stdio.h>\n#include "jackpot.h"\nint main(void){printf("%d %d %d %d %d %d", JP_W4_MAX_TOKENS, '
                   'JP_VERIFY_MAX_DRAFT, JP_NORM_RMS, JP_BF16, JP_F32, JP_F16);return 0;}\n')
    exe = tmp_path / "lim"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [B.JP_W4_MAX_TOKENS, B.JP_VERIFY_MAX_DRAFT, B.JP_NORM_RMS, B.JP_BF16, B.JP_F32, B.JP_F16]


def test_calls_without_a_context_are_refused():
    jp_build.build()
    lib = B.load()
    n, w, v = B.jp_norm_desc(T=1, H=8), B.jp_w4_desc(N=1, K=8, group=32), B.jp_verify_desc(B=1, V=8)
    assert lib.jp_layer_norm_forward(None, ctypes.byref(n), *[None] * 6) == -1
    assert lib.jp_layer_norm_backward(None, ctypes.byref(n), *[None] * 9, 0) == -1
    assert lib.jp_layer_norm_workspace_bytes(None, 1, 8, 0) == 0
    assert lib.jp_w4_pack(None, ctypes.byref(w), None, None, None, None) == -1
    assert lib.jp_w4_linear(None, ctypes.byref(w), None, None, 0, 1, None, 0, 0) == -1
    assert lib.jp_verify_draft(None, ctypes.byref(v), *[None] * 12, 0) == -1
    assert lib.jp_verify_workspace_bytes(None, 1, 1, 8, 0, 1) == 0


def test_a_wrong_dtype_is_refused_by_the_arguments_name():
    """The checks of dtypes come before anything that needs a device."""
    class Ctx:
        _descs = {}
    x, w = torch.empty((2, 8), dtype=torch.float16), torch.empty(8)
    with pytest.raises(B.JackpotError, match="^x must be bfloat16 or float32"):
        runner.layer_norm(Ctx(), x, w)
    with pytest.raises(B.JackpotError, match="^weight must be bfloat16 or float32"):
        runner.layer_norm(Ctx(), x.float(), w.half())
    packed = runner.W4Weight(torch.empty(0, dtype=torch.uint8), 4, 8, 32)
    with pytest.raises(B.JackpotError, match="^out must be bfloat16 or float32"):
        runner.linear_w4(Ctx(), x.bfloat16(), packed, out_dtype=torch.float16)
    with pytest.raises(B.JackpotError, match="^logits must be bfloat16 or float32"):
        B._dtype_code(x)
