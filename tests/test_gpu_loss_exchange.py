"""The wait of blocks that share a row of logits, where it gives up."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("limit", [1, 20_000_000])
def test_a_part_that_comes_too_late_finds_the_block_that_gave_up(limit):
    """The second launch of the self-test: one of two blocks sends its part behind the other one's limit.  The status reads the first launch's
    JP_ERR_TIMEOUT (JP_ERR_CUDA if the part was lost or a block read a wrong total), and the context works as before."""
    jp_build.build()
    ctx = B.Context(0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = ctx.launch_count()
    B.jp_selftest_bounded_wait(ctx, limit, status)
    assert ctx.launch_count() == before + 2
    torch.cuda.synchronize()
    assert status.item() == -6
    z = torch.randn((2, 151936), device="cuda").bfloat16()   # eight blocks a row
    tok, one = torch.tensor([5, 7], dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, tok.long()[:, None])[:, 0]
    o = runner.policy_loss(ctx, z, tok, one, lp.float(), eps_lo=0.0, eps_hi=0.0)
    assert (o["state"] == 1).all() and ((o["logp"].double() - lp).abs() < 2e-5).all() and abs(float(o["loss"][0]) + 1) < 4e-5
    ctx.close()
