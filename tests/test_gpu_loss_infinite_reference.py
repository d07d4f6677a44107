"""Pairs whose reference gives one sequence the probability 0: h is infinite, the loss 0 or infinite, and the other pairs as without them."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


# the side that the reference rules out, and the loss: chosen: h = inf, -log sigma(h) = 0; rejected: h = -inf
@pytest.mark.parametrize("side,smoothing,finite", [(0, 0.0, True), (1, 0.0, False), (0, 0.1, False), (1, 1.0, True), (0, 1.0, False), (1, 0.1, False)])
def test_a_sequence_without_probability_in_the_reference(ctx, side, smoothing, finite):
    g = torch.Generator(device="cuda").manual_seed(2)
    z = torch.randn((10, 300), generator=g, device="cuda")
    tok = torch.randint(0, 300, (10,), generator=g, device="cuda").int()
    start = torch.tensor([0, 3, 5, 7, 10], dtype=torch.int32, device="cuda")
    ref = torch.tensor([-12.0, -11.0, -10.0, -14.0], device="cuda")
    clean = runner.preference_loss(ctx, z, tok, start, ref_logp=ref, label_smoothing=smoothing)
    alone = runner.preference_loss(ctx, z[5:], tok[5:], start[2:] - 5, ref_logp=ref[2:], label_smoothing=smoothing)
    ref[side] = -INF
    o = runner.preference_loss(ctx, z, tok, start, ref_logp=ref, label_smoothing=smoothing)
    assert o["margin"][0] == (INF if side == 0 else -INF) and o["margin"][1] == clean["margin"][1]
    assert torch.equal(o["d_logits"][5:], clean["d_logits"][5:])
    if finite:                                   # half of the other pair's loss, rounded once; and nothing to learn from the pair
        assert abs(float(o["loss"]) - float(alone["loss"]) / 2) <= 2.0 ** -23 * float(alone["loss"]) and (o["d_logits"][:5] == 0).all()
    else:
        assert float(o["loss"]) == INF and o["d_logits"].isfinite().all()
