"""The structs of the losses, the block norms and the 8-bit layers as gcc sees them in the header against their ctypes mirrors, and what
those calls answer without a context or with sizes out of range (no device is needed)."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"jp_policy_desc": B.jp_policy_desc, "jp_preference_desc": B.jp_preference_desc, "jp_block_norm_desc": B.jp_block_norm_desc,
           "jp_i8_desc": B.jp_i8_desc}


def compiled(tmp_path, body):
    src, exe = tmp_path / "p.c", tmp_path / "p"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "jackpot.h"\nint main(void){' + body + 'return 0;}\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    return [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]


def test_structs_match_the_header(tmp_path):
    got = compiled(tmp_path, "".join(f'printf("%zu ", sizeof({n}));' + "".join(f'printf("%zu ", offsetof({n}, {f}));' for f, _ in c._fields_)
                                     for n, c in STRUCTS.items()))
    want = []
    for c in STRUCTS.values():
        want += [ctypes.sizeof(c)] + [getattr(c, f).offset for f, _ in c._fields_]
    assert got == want


def test_constants_match_the_header(tmp_path):
    assert compiled(tmp_path, 'printf("%d %d", JP_PREFERENCE_AVERAGE, JP_I8_MAX_K);') == [B.JP_PREFERENCE_AVERAGE, B.JP_I8_MAX_K]


def test_calls_without_a_context_are_refused():
    jp_build.build()
    lib = B.load()
    p, q, n, w = B.jp_policy_desc(T=1, V=8), B.jp_preference_desc(T=1, V=8, P=0), B.jp_block_norm_desc(T=1, H=8), B.jp_i8_desc(N=1, K=8)
    assert lib.jp_policy_loss(None, ctypes.byref(p), *[None] * 13, 0) == -1
    assert lib.jp_preference_loss(None, ctypes.byref(q), *[None] * 12, 0) == -1
    assert lib.jp_block_norm_forward(None, ctypes.byref(n), *[None] * 14) == -1
    assert lib.jp_block_norm_backward(None, ctypes.byref(n), *[None] * 22, 0) == -1
    assert lib.jp_i8_pack(None, ctypes.byref(w), None, None, None) == -1
    assert lib.jp_i8_quantize(None, None, 0, 1, 8, None, 0) == -1
    assert lib.jp_i8_linear(None, ctypes.byref(w), None, None, 0, 1, None, 0, None, 0, 0, None) == -1
    assert lib.jp_policy_workspace_bytes(None, 1) == lib.jp_preference_workspace_bytes(None, 1, 1) == lib.jp_block_norm_workspace_bytes(None, 1, 8, 0) == 0


def test_sizes_of_8_bit_buffers():
    """128 channels x 128 features a tile, 8 tokens a group, and a scale each; 0 for what there is no layout of."""
    assert B.jp_i8_packed_bytes(1, 1) == 128 * 128 + 128 * 4
    assert B.jp_i8_packed_bytes(129, 200) == 2 * 2 * 128 * 128 + 2 * 128 * 4
    assert B.jp_i8_token_bytes(1, 1) == 8 * 128 + 8 * 4 and B.jp_i8_token_bytes(17, 129) == 24 * 256 + 24 * 4
    for n, k in ((0, 1), (1, 0), (1, B.JP_I8_MAX_K + 1), (1 << 31, 1), (-1, 5)):
        assert B.jp_i8_packed_bytes(n, k) == 0
    assert B.jp_i8_token_bytes(0, 1) == B.jp_i8_token_bytes(1 << 24, 1) == B.jp_i8_token_bytes(1, 0) == 0
    for m, k in ((1, 1), (8, 128), (9, 129), (777, 1111), (3, 65536)):       # the runner's own arithmetic
        data, _ = runner._token_buffer(torch.empty((m, k), dtype=torch.bfloat16))
        assert data.numel() == B.jp_i8_token_bytes(m, k)


def test_refusals_before_a_device_is_needed():
    class Ctx:
        _descs = {}
    z, tok, f = torch.empty((4, 8), dtype=torch.float16), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    with pytest.raises(B.JackpotError, match="^logits must be bfloat16 or float32"):
        runner.policy_loss(Ctx(), z, tok, f, f)
    with pytest.raises(B.JackpotError, match="^tokens must be"):
        runner.preference_loss(Ctx(), z.float(), tok.long(), tok[:3])
    with pytest.raises(B.JackpotError, match="^seq_start must be"):
        runner.preference_loss(Ctx(), z.float(), tok, tok[:2])
    with pytest.raises(B.JackpotError, match="^weight must be bfloat16 or float32"):
        runner.block_norm(Ctx(), z.float(), z.float(), torch.empty(8, dtype=torch.float16))
    with pytest.raises(B.JackpotError, match="^gate must be"):
        runner.block_norm(Ctx(), z.float(), z.float(), torch.empty(8), gate=torch.empty(7))
    with pytest.raises(B.JackpotError, match="^rstd is missing"):
        runner.block_norm_backward(Ctx(), z.float(), None, z.float(), z.float(), torch.empty(8), None, None, rms=True)
    with pytest.raises(B.JackpotError, match="^x must be bfloat16"):
        runner.linear_i8(Ctx(), z, runner.I8Weight(torch.empty(0, dtype=torch.uint8), 4, 8))


def test_weights_round_to_the_nearest_step():
    w = torch.tensor([[1.0, -2.0, 0.5, 0.0], [0.0, 0.0, 0.0, 0.0]])
    q, s = runner.quantize_i8(w)
    assert q.tolist() == [[64, -127, 32, 0], [0, 0, 0, 0]] and float(s[1]) == 0.0 and abs(float(s[0]) - 2 / 127) < 1e-8
