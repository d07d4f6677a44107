"""The policy loss's KL term next to 0, where the policy is the reference: k = exp(d) - d - 1 is d^2 / 2 there, and never below 0.

Bars.  One entry of logit 0 has lp = 0 exactly, so d is logp_ref itself: k is fp64 up to 2^-32 of itself (the difference of exp(d) - 1 and d, from
|d| = 2^-10 on) and rounded to fp32 once; the gradient's coefficient is -kl_coef (exp(d) - 1), of which p (1 - p) = 0 leaves nothing, so it is held
over two entries, where the sums of exponentials err by 2^-22 each way."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def test_next_to_zero(ctx):
    n = 4000
    d = torch.logspace(-14, 0.5, n, dtype=torch.float64).float().cuda()
    d = torch.cat([d, -d, torch.zeros(1, device="cuda"), torch.tensor([2.0 ** -10, -2.0 ** -10], device="cuda")])
    T = d.numel()
    z, tok, zero = torch.zeros((T, 4), device="cuda")[:, :1], torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, device="cuda")
    o = runner.policy_loss(ctx, z, tok, zero, zero, logp_ref=d, kl_coef=1.0)
    x = d.double()
    want = torch.where(x.abs() < 0.01, x * x * (0.5 + x / 6 + x * x / 24 + x ** 3 / 120 + x ** 4 / 720 + x ** 5 / 5040), torch.expm1(x) - x)
    assert (o["logp"] == 0).all() and (o["kl"] >= 0).all()
    assert ((o["kl"].double() - want).abs() <= (U + 2.0 ** -32) * want + 2.0 ** -149).all()
    assert (o["loss"][2].double() - want.mean()).abs() <= 2 * U * want.mean()


@pytest.mark.parametrize("grad", [True, False])
def test_a_reference_that_is_the_policy(ctx, grad):
    """The ordinary first step: logp_ref is the call's own logp, so d is a rounding to fp32, at most U |lp| (and what lp errs by is in both)."""
    T, V = 3000, 1200
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((T, V), generator=g, device="cuda")
    tok = torch.randint(0, V, (T,), generator=g, device="cuda")
    z.scatter_(1, tok[:, None], 20 * torch.rand((T, 1), generator=g, device="cuda"))     # from certain to unlikely
    tok, zero = tok.int(), torch.zeros(T, device="cuda")
    own = runner.policy_loss(ctx, z, tok, zero, zero, grad=grad)["logp"]
    o = runner.policy_loss(ctx, z, tok, zero, zero, logp_ref=own, kl_coef=0.1, grad=grad)
    assert torch.equal(o["logp"], own) and (own.abs() < 0.1).any() and (own.abs() > 5).any()
    assert (o["kl"] >= 0).all() and (o["loss"][2] >= 0) and (o["kl"].double() <= 0.51 * (U * own.double().abs()) ** 2 + 2.0 ** -149).all()


def test_gradient_next_to_zero(ctx):
    """Two equal entries: dL/dz = -kl_coef (exp(d) - 1) (+-1/2) / T."""
    d = torch.logspace(-12, -1, 500, dtype=torch.float64).float().cuda()
    d = torch.cat([d, -d])
    T = d.numel()
    ln2 = torch.log(torch.tensor(2.0, dtype=torch.float64))
    ref = (d.double().cpu() - ln2).float().cuda()             # lp = -ln 2 within 2 U; d as it comes out
    z, tok, zero = torch.zeros((T, 4), device="cuda")[:, :2], torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, device="cuda")
    o = runner.policy_loss(ctx, z, tok, zero, zero, logp_ref=ref, kl_coef=1.0)
    want = -torch.expm1(ref.double() + ln2.item()) / 2 / T
    assert ((o["d_logits"][:, 0].double() - want).abs() <= 2.0 ** -20 * want.abs() + 4 * U / T).all()
    assert ((o["d_logits"][:, 0] + o["d_logits"][:, 1]).abs() <= 2.0 ** -20 * want.abs() + 4 * U / T).all()
