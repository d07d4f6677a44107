"""The losses over long rows that one block streams (more rows than SMs, no gradient kept in shared memory), and that blocks read twice.

Bars.  Those of the losses' other tests, with the number of additions that these rows take: a thread adds one vector of 4 (fp32) or 8 (bf16) terms at a
time, n = ceil(V / 4 / 512) = 489 or ceil(V / 8 / 512) = 245, each off by u of the sum so far, so by n u / 2 in all for terms of one distribution; X = 2^-22
of a term's 2^x, its exponent's rounding, the tree of a vector and each of 15 merges: 16 X + 10 u.  489 / 2 u + 16 X + 10 u < 1.9e-5."""
import pytest
import torch

import test_gpu_loss as base
from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_million_entries(ctx, dtype, monkeypatch):
    monkeypatch.setattr(base, "E", 1.9e-5 + 1.34e-8 * 14)    # (log2(e) in fp32: 1.34e-8 of the row's entropy, below ln V)
    T, V = 160, 1_000_001
    z, tok, adv, old, ref, mask, weight = base.make(T, V, dtype, 3)
    P = base.plain_policy(z, tok, adv, old, ref, mask, weight, 0, 0.2, 0.28, 0.05, 1.0, 1.0)
    args = dict(logp_ref=ref, mask=mask, token_weight=weight, eps_lo=0.2, eps_hi=0.28, kl_coef=0.05)
    base.check_policy(runner.policy_loss(ctx, z, tok, adv, old, grad=False, **args), dtype, P, 0.05, grad=False)
    base.check_policy(runner.policy_loss(ctx, z, tok, adv, old, **args), dtype, P, 0.05)
    del P
    start = torch.tensor([0, 60, 90, 100, 160], dtype=torch.int32, device="cuda")
    P = base.plain_preference(z, tok, start, None, mask, 0.1, 0.1, 0.0, False, 1.0)
    base.check_preference(runner.preference_loss(ctx, z, tok, start, mask=mask, beta=0.1, label_smoothing=0.1), dtype, P)
