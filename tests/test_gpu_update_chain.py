"""The operators one after the other as a program uses them: a quantised model's last block over a prompt (norms, 8-bit projection, gate, 8-bit
output layer), the losses on its logits, and the gradient back through the norms; each against what the steps give in 64 bits."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def model(H, V, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")
    return dict(proj=r(H, H) / H ** 0.5, head=r(V, H) * 2 / H ** 0.5, first=(1 + 0.1 * r(H)).to(BF), post=(1 + 0.1 * r(H)).to(BF),
                last=(1 + 0.1 * r(H)).to(BF), gate=(0.5 + 0.1 * r(H)).to(BF))


def rms64(x, w):
    return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6) * w.double()


def test_update_through_a_quantised_block(ctx):
    T, H, V = 90, 256, 3001
    m = model(H, V, 1)
    proj, head = (runner.pack_i8(ctx, *runner.quantize_i8(m[k])) for k in ("proj", "head"))
    g = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn((T, H), generator=g, device="cuda").to(BF)
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8)
    adv = torch.randn(T, generator=g, device="cuda")

    def forward():
        x, _, _ = runner.layer_norm(ctx, h, m["first"], rms=True)
        o = runner.linear_i8(ctx, x, proj)
        f = runner.block_norm(ctx, o, h, m["last"], post_weight=m["post"], gate=m["gate"], scale=0.5, rms=True)
        logits = runner.linear_i8(ctx, f["y"], head, out=torch.empty((T, (V + 7) // 8 * 8), device="cuda", dtype=BF)[:, :V])
        return o, f, logits
    o, f, logits = forward()
    # the block in 64 bits, with the 8-bit weights as they are: rounding x to 8 bits is off by half a step of 1 / 127 of the row's largest
    # entry, and bf16 by 2^-8 at each of four places; both average over 256 products
    y = rms64(h.double(), m["first"])
    dq = lambda w: (runner.quantize_i8(w)[0].double() * runner.quantize_i8(w)[1].double()[:, None])
    y = rms64(h.double() + 0.5 * m["gate"].double() * rms64(y @ dq(m["proj"]).t(), m["post"]), m["last"])
    want = y @ dq(m["head"]).t()
    assert float((logits.double() - want).norm() / want.norm()) < 0.02

    old = torch.log_softmax(logits.double(), 1).gather(1, tok.long()[:, None])[:, 0].float()
    p = runner.policy_loss(ctx, logits, tok, adv, old, logp_ref=old, mask=mask, kl_coef=0.1)
    # where old and reference are the model itself the loss is -mean(A) and its gradient -A (1[v = x] - p) / N
    n = int(mask.sum())
    on = mask.double()
    assert abs(float(p["loss"][0]) + float((adv.double() * on).sum() / n)) < 1e-5
    soft = torch.softmax(logits.double(), 1)
    hot = torch.zeros_like(soft).scatter_(1, tok.long()[:, None], 1.0)
    d = -(adv.double() * on / n)[:, None] * (hot - soft)
    assert float((p["d_logits"].double() - d).norm() / d.norm()) < 2.0 ** -8 + 1e-4

    # back through the output layer (its product in torch) and the norms; the residual stream gets its own gradient besides
    dy = (p["d_logits"].float() @ dq(m["head"]).float()).to(BF)
    b = runner.block_norm_backward(ctx, dy, None, o, f["sum"], m["last"], None, f["rstd"], post_weight=m["post"], post_rstd=f["post_rstd"],
                                   gate=m["gate"], scale=0.5, rms=True, bias=False)
    x64, s64 = o.double().requires_grad_(True), f["sum"].double().requires_grad_(True)
    gate, last, post = (m[k].double().requires_grad_(True) for k in ("gate", "last", "post"))
    ds = torch.autograd.grad((rms64(s64, last) * dy.double()).sum(), [s64, last])
    dx = torch.autograd.grad((0.5 * gate * rms64(x64, post) * ds[0]).sum(), [x64, gate, post])
    for got, ref in ((b["dresidual"], ds[0]), (b["dweight"], ds[1]), (b["dx"], dx[0]), (b["dgate"], dx[1]), (b["dpost_weight"], dx[2])):
        assert float((got.double() - ref).norm() / ref.norm()) < (2.0 ** -8 if got.dtype is BF else 1e-5)

    # the same calls captured, replayed on new hidden states
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o2, f2, l2 = forward()
        p2 = runner.policy_loss(ctx, l2, tok, adv, old, logp_ref=old, mask=mask, kl_coef=0.1, d_logits=l2)
    h.copy_(h.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(f2["y"], f["y"].flip(0)) and torch.equal(o2, o.flip(0))
    h.copy_(h.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(l2, p["d_logits"]) and torch.equal(p2["loss"], p["loss"])


def test_preference_beside_the_policy_loss(ctx):
    """The two losses read the same rows: equal log-probabilities, and the reference's sums come from the other call's outputs."""
    T, V = 60, 2000
    g = torch.Generator(device="cuda").manual_seed(4)
    z = (torch.randn((T, V), generator=g, device="cuda") * 3).to(BF)
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    zero = torch.zeros(T, device="cuda")
    start = torch.tensor([0, 20, 33, 50, 60], dtype=torch.int32, device="cuda")
    p = runner.policy_loss(ctx, z, tok, zero, zero, grad=False)
    first = runner.preference_loss(ctx, z, tok, start, grad=False)
    assert torch.equal(p["logp"], first["logp"])
    again = runner.preference_loss(ctx, z, tok, start, ref_logp=first["seq_logp"], beta=0.3)
    # the reference is the model itself up to the rounding of its sums to fp32: h is 0 and the loss log 2
    assert (again["margin"].abs() <= 0.3 * 4 * 2.0 ** -24 * first["seq_logp"].abs().max()).all()
    assert abs(float(again["loss"]) - 0.6931471805599453) < 1e-4
    half = torch.zeros(T, device="cuda")
    for i in range(2):
        a, b, c = (int(start[2 * i + j]) for j in range(3))
        half[a:b], half[b:c] = -0.3 / 4, 0.3 / 4
    soft = torch.softmax(z.double(), 1)
    hot = torch.zeros_like(soft).scatter_(1, tok.long()[:, None], 1.0)
    d = half.double()[:, None] * (hot - soft)
    assert float((again["d_logits"].double() - d).norm() / d.norm()) < 2.0 ** -8 + 1e-4
