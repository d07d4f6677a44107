"""Block norms of narrow rows that start off 16 bytes, packed so that a 16-byte vector holds several of them and reaches beyond the matrix from more
rows than the first and the last, beside NaN: against the plain implementation in 64 bits and its bars, which hold for rows of up to 16 terms a thread."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner
from test_gpu_block_norm import arguments, check_backward, check_forward, make

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("T", [1, 2, 3, 10, 1000])
@pytest.mark.parametrize("H,ld", [(1, 1), (2, 3), (3, 3), (5, 5), (7, 7), (3, 11)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("same", [True, False])
def test_narrow_rows_at_odd_starts(ctx, T, H, ld, dtype, same):
    """``same``: all matrices at one offset to 16 bytes, or each at its own."""
    for start in (1, 3):
        s = make(T, H, dtype, F32, "all", T * 100 + H, ld, start)
        if not same:
            for k, off in (("x", 2), ("dy", 5)):
                flat = torch.full((off + T * ld,), float("nan"), device="cuda", dtype=dtype)
                m = flat[off:].view(T, ld)[:, :H]
                m.copy_(s[k])
                s[k] = m
        for rms in (True, False):
            f = runner.block_norm(ctx, s["x"], s["residual"], s["weight"], s["bias"], eps=1e-6, rms=rms, **arguments(s))
            check_forward(f, s, rms, s["residual"])
            total = torch.full((start + T * ld,), float("nan"), device="cuda", dtype=dtype)[start:].view(T, ld)[:, :H]
            total.copy_(f["sum"])
            o = runner.block_norm_backward(ctx, s["dy"], s["dsum"], s["x"], total, s["weight"], f["mean"], f["rstd"], post_mean=f["post_mean"],
                                           post_rstd=f["post_rstd"], rms=rms, **arguments(s))
            check_backward(o, s, f, total, rms, s["dsum"])
