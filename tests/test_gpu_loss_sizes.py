"""The losses at vocabularies between the steps of the launch plan: 13 and 14 vectors a thread, 256 and 512 threads, one to eight blocks a row, and
as many rows as make the blocks take several."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from test_gpu_loss import test_policy_matches_the_formula as policy_matches

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("T,V,dtype", [(1500, 24000, BF), (700, 26627, BF), (700, 28672, BF), (1500, 12001, F32), (700, 14335, F32), (700, 24001, F32), (700, 50257, BF),
                                       (300, 50257, F32), (700, 56001, BF), (350, 100277, BF), (170, 200064, BF), (160, 228000, BF), (160, 335000, BF), (8, 400003, BF),
                                       (8, 200001, F32)])
def test_vocabularies_between_the_steps(ctx, T, V, dtype):
    for form in ("all", "bare"):
        policy_matches(ctx, T, V, dtype, form)
