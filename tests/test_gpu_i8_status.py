"""The status of an 8-bit linear layer, through the runner."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner
from test_gpu_i8 import check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("M", [0, 1, 5, 300])
def test_status_is_written_by_every_call(ctx, M):
    x, q, scales = make(M, 130, 200, 1)
    w = runner.pack_i8(ctx, q, scales)
    for tokens in (x, runner.quantize_tokens_i8(ctx, x)):
        status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
        out = runner.linear_i8(ctx, tokens, w, out_dtype=torch.float32, status=status)
        assert status.item() == 0
        check(out, x, q, scales)


def test_refusals(ctx):
    x, q, scales = make(2, 16, 16, 1)
    w = runner.pack_i8(ctx, q, scales)
    for status in (torch.zeros(1, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")):
        with pytest.raises(B.JackpotError, match="status must be"):
            runner.linear_i8(ctx, x, w, status=status)
    with pytest.raises(B.JackpotError, match="context is on"):
        runner.linear_i8(ctx, x, w, status=torch.zeros(1, dtype=torch.int32))
