"""8-bit linear layers whose scales lie at the ends of fp32: the product of the two scales leaves the normal numbers where the output does not.

Bars.  As in the layers' other tests, 4.01 u for the scale of a token, the product of the scales, the sum as fp32 and their product, and half a step of
the output's type: of the value, or of the smallest normal number where the output lies below it.  Tokens are chosen so that their scales are normal
numbers."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner
from test_gpu_i8 import rounded

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


# one launch for one token; K shared by a cluster; channels dealt evenly; tiles; pairs of CTAs
@pytest.mark.parametrize("M,N,K", [(1, 640, 256), (5, 130, 640), (48, 20000, 128), (300, 12000, 128), (700, 16384, 128)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("power,scale", [(-100, 1e-12), (-115, 3e-4), (-100, 2e-45), (-60, 1e-38), (0, 1e-45), (125, 200.0), (125, 1e-44), (120, 3e38), (100, 1e-10)])
def test_scales_at_the_ends_of_fp32(ctx, M, N, K, dtype, power, scale):
    g = torch.Generator(device="cuda").manual_seed(M)
    x = (torch.randn((M, K), generator=g, device="cuda").clamp(-3.5, 3.5).double() * 2.0 ** power).to(BF)
    q = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    q[::3] = 0                                   # sums of 0: 0, whatever the scales
    scales = (scale * (0.5 + torch.rand(N, generator=g, device="cuda").double() / 2)).float()
    scales[1::2] *= -1
    if M > 2:
        x[1] = 0
    out = runner.linear_i8(ctx, x, runner.pack_i8(ctx, q, scales), out_dtype=dtype)
    xq, sx = rounded(x)
    want = (xq @ q.double().t()) * sx * scales.double()
    assert (out[:, ::3] == 0).all() and (M <= 2 or (out[1] == 0).all())
    most = torch.finfo(dtype).max
    beyond = want.abs() > most
    half = 2.0 ** -8 if dtype is BF else U
    near = (want.abs() > most * (1 - 2 * half)) & ~beyond     # may round to infinity
    # (below 2^-126 the step of fp32 is 2^-149, so its rounding is off by 2^-150, more than u of the value; that of bf16 comes on top of it)
    bar = 4.01 * U * want.abs() + 2.0 ** -150 + half * want.abs().clamp(min=2.0 ** -126)
    good = ((out.double() - want).abs() <= bar) | (beyond & (out.double() == want.sign() * float("inf"))) | (beyond & (out.double().abs() >= most * (1 - 2 * half)))
    assert (good | (near & out.isinf())).all()
