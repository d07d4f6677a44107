"""The losses' gradient times an upstream scalar, 0 among them: an auxiliary loss annealed to nothing trains nothing."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-60, 1.0, -2.0])
@pytest.mark.parametrize("in_place", [False, True])
def test_the_upstream_scalar(ctx, scale, in_place):
    T, V = 6, 500
    g = torch.Generator(device="cuda").manual_seed(1)
    wide = torch.randn((T, V + 4), generator=g, device="cuda")
    tok = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    f = torch.randn(T, generator=g, device="cuda")
    start = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")
    policy = lambda z, **k: runner.policy_loss(ctx, z, tok, f, f - 4, eps_lo=0.0, eps_hi=0.0, **k)
    preference = lambda z, **k: runner.preference_loss(ctx, z, tok, start, **k)
    for loss in (policy, preference):
        one = loss(wide[:, :V])
        rows = wide.clone()
        z = rows[:, :V]
        got = loss(z, grad_out=scale, d_logits=z if in_place else None)
        assert torch.equal(got["loss"], one["loss"]) or abs(float(scale)) < 1e-45 and torch.allclose(got["loss"], one["loss"], rtol=1e-5)
        # a power of two times the gradient, or nothing
        assert torch.equal(got["d_logits"], one["d_logits"] * (scale if abs(scale) > 1e-45 else 0.0)) and (one["d_logits"] != 0).any()
        assert got["d_logits"].shape == (T, V) and torch.equal(rows[:, V:], wide[:, V:])
