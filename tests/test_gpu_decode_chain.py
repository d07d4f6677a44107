"""The operators around the output layer one after the other, as a rollout and a training step use them: last norm, output layer
with 4-bit weights, verification of drafted tokens, the record for the OBRS pass, and the norm's backward with the gradient that
comes back through the output layer.  Also: offsets beyond 32 bits in each of them.

Bars are those of the operators' own tests (test_gpu_norm.py, test_gpu_w4.py, test_gpu_verify.py)."""

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


def dequantised(q, s, z, K, group):
    v = torch.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1)[:, :K].double()
    grp = torch.arange(K, device=q.device) // group
    return (v - (8.0 if z is None else z.double()[:, grp])) * s.double()[:, grp]


def test_rollout_step_and_its_record(ctx):
    n_seq, N, H, V, group = 6, 3, 256, 2048, 64
    g = torch.Generator(device="cuda").manual_seed(21)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    gain = (1 + 0.1 * rnd(H)).to(torch.bfloat16)
    ht, hd = rnd(n_seq * (N + 1), H).to(torch.bfloat16), rnd(n_seq * N, H).to(torch.bfloat16)
    hd.view(n_seq, N, H).copy_((ht.view(n_seq, N + 1, H)[:, :N].float() + 0.3 * rnd(n_seq, N, H)).to(torch.bfloat16))
    q, s, z = runner.quantize_w4((rnd(V, H) * 0.2), group, symmetric=False)
    w = runner.pack_w4(ctx, q, s, z, K=H, group=group)
    logits = []
    for h in (ht, hd):
        y, _, rstd = runner.layer_norm(ctx, h, gain, eps=1e-6, rms=True)
        out = runner.linear_w4(ctx, y, w, out_dtype=torch.bfloat16)
        wd = dequantised(q, s, z, H, group)
        ref, mag = y.double() @ wd.t(), y.double().abs() @ wd.abs().t()
        assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (48 + H / group) * U * mag).all()
        logits.append(out)
    target, draft = logits[0].view(n_seq, N + 1, V), logits[1].view(n_seq, N, V)
    noise = -torch.log(-torch.log(torch.rand((n_seq, N, V), generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    tokens = (draft.float() + noise).argmax(2).to(torch.int32)
    out = runner.verify_draft(ctx, target, draft, tokens, torch.rand((n_seq, N), generator=g, device="cuda"),
                              torch.rand(n_seq, generator=g, device="cuda"))
    n_acc, emitted = out["n_accepted"].cpu(), out["tokens"].cpu()
    logp = torch.log_softmax(target.double(), 2)
    rows = [(b, i) for b in range(n_seq) for i in range(int(n_acc[b]) + 1)]
    for b, i in rows:
        x = int(emitted[b, i])
        assert 0 <= x < V and (i == int(n_acc[b]) or x == int(tokens[b, i]))
        assert abs(float(out["logp"][b, i]) - float(logp[b, i, x])) <= 6e-6 + U * abs(float(logp[b, i, x]))
    # the record goes to the pass that corrects for the rollout model: acceptance from the stored log-probabilities
    at = torch.tensor([b * (N + 1) + i for b, i in rows], device="cuda")
    tok = out["tokens"].reshape(-1)[at].contiguous()
    logp_inf = out["logp"].reshape(-1)[at].contiguous()
    policy = (target.reshape(-1, V)[at].float() + 0.5 * rnd(len(rows), V)).to(torch.bfloat16)
    top = torch.log_softmax(target.reshape(-1, V)[at].float(), 1).topk(20)
    rec = runner.forward_sparse_actor(ctx, policy, tok, None, logp_inf, top.indices.to(torch.int32).contiguous(),
                                      top.values.contiguous(), lam=1.5, k=16, seed=9)
    lp = torch.log_softmax(policy.double(), 1).gather(1, tok.long()[:, None])[:, 0]
    want = torch.exp(lp - logp_inf.double()).div(1.5).clamp(max=1)
    assert ((rec["accept_prob"].double() - want).abs() <= 2e-5 * want + 1e-7).all()
    assert rec["stats"]["n_valid"] == len(rows)


def test_training_step_through_the_norm(ctx):
    """jp_obrs_backward's gradient of the policy logits, back through the output layer into the norm."""
    T, H, V = 96, 512, 4096
    g = torch.Generator(device="cuda").manual_seed(22)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    h, gain, shift = rnd(T, H).to(torch.bfloat16), 1 + 0.1 * rnd(H), 0.1 * rnd(H)
    wp = (rnd(V, H) * 0.15).to(torch.bfloat16)
    y, mean, rstd = runner.layer_norm(ctx, h, gain, shift, eps=1e-5)
    zp = (y.float() @ wp.float().t()).to(torch.bfloat16)
    za = (zp.float() + 0.4 * rnd(T, V)).to(torch.bfloat16)
    tok = torch.multinomial(za.float().softmax(1), 1, generator=g)[:, 0].to(torch.int32)
    fwd = runner.forward(ctx, za, zp, tok, lam=1.5, k=16, seed=4)
    adv = rnd(T)
    _, dzp = runner.backward(ctx, za, zp, tok, None, fwd["accept"], fwd["weight"], advantages=adv)
    dy = (dzp.float() @ wp.float()).to(torch.bfloat16)
    dx, dw, db = runner.layer_norm_backward(ctx, dy, h, gain, mean, rstd)
    x, d, r = h.double(), dy.double(), rstd.double()[:, None]
    xh = (x - mean.double()[:, None]) * r
    gg = d * gain.double()
    ref = (gg - gg.mean(1, keepdim=True) - xh * (gg * xh).mean(1, keepdim=True)) * r
    mag = (gg.abs() + gg.abs().mean(1, keepdim=True) + xh.abs() * (gg * xh).abs().mean(1, keepdim=True)) * r
    assert ((dx.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 64 * U * mag).all()
    loss = (d.abs() * (x.abs() + mean.double().abs()[:, None]) * r).sum(0)
    assert ((dw.double() - (d * xh).sum(0)).abs() <= 128 * U * (d * xh).abs().sum(0) + 4 * U * loss).all()
    assert ((db.double() - d.sum(0)).abs() <= 128 * U * d.abs().sum(0)).all()
    assert float(dw.abs().sum()) > 0


def test_two_streams_at_once(ctx):
    """Calls of one context on two streams, and graphs replayed on both, do not share scratch."""
    g = torch.Generator(device="cuda").manual_seed(23)
    V, N, n = 30011, 4, 24
    cases = []
    for i in range(2):
        z = (torch.randn((n, N + 1, 30016), generator=g, device="cuda") * 2.5).to(torch.bfloat16)[:, :, :V]
        d = (z[:, :N].float() + 0.6 * torch.randn((n, N, V), generator=g, device="cuda")).to(torch.bfloat16)
        dp = torch.zeros((n, N, 30016), dtype=torch.bfloat16, device="cuda")
        dp[:, :, :V] = d
        tok = torch.randint(0, V, (n, N), generator=g, device="cuda", dtype=torch.int32)
        cases.append((z, dp[:, :, :V], tok, torch.rand((n, N), generator=g, device="cuda") * 0.01,
                      torch.rand(n, generator=g, device="cuda")))
    want = [{k: v.clone() for k, v in runner.verify_draft(ctx, *c).items()} for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(runner.verify_draft(ctx, *cases[i]))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            outs.append(runner.verify_draft(ctx, *cases[i]))
        graphs.append(gr)
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for i in range(2):
        for o in got[i] + [outs[i]]:
            assert all(torch.equal(o[k], want[i][k]) for k in want[i])


def test_norm_rows_beyond_32_bit_offsets(ctx):
    T, H = 560000, 4096                          # 2.3e9 elements
    x = torch.zeros((T, H), dtype=torch.bfloat16, device="cuda")
    tail = (torch.randn((5, H), device="cuda") + 0.5).to(torch.bfloat16)
    x[-5:] = tail
    w, b = torch.rand(H, device="cuda") + 0.5, torch.rand(H, device="cuda")
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=1e-6)
    y5, m5, r5 = runner.layer_norm(ctx, tail, w, b, eps=1e-6)
    ref = (tail.double() - m5.double()[:, None]) * r5.double()[:, None] * w.double() + b.double()
    assert ((y[-5:].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 64 * U * (ref.abs() + 2 * b.double() + 8)).all()
    assert torch.equal(y[0], b.to(torch.bfloat16)) and torch.equal(y[T - 6], y[0])
    assert ((mean[-5:] - m5).abs() <= 64 * U * tail.float().abs().mean(1)).all()
    del y
    dx, dw, db = runner.layer_norm_backward(ctx, x, x, w, mean, rstd, dx=x)       # dy = x, in its place
    xd, m, r = tail.double(), mean[-5:].double()[:, None], rstd[-5:].double()[:, None]
    xh = (xd - m) * r
    assert ((dw.double() - (xd * xh).sum(0)).abs() <= 128 * U * (xd * xh).abs().sum(0) + 16 * U * (xd.abs() * (xd.abs() + 1) * r).sum(0)).all()
    assert ((db.double() - xd.sum(0)).abs() <= 128 * U * xd.abs().sum(0)).all()
    g = xd * w.double()
    want = (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True)) * r
    mag = (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True)) * r
    assert ((dx[-5:].double() - want).abs() <= 2.0 ** -8 * want.abs() + 64 * U * mag).all()
    assert (dx[:3] == 0).all() and (dx[T - 6] == 0).all()


def test_verify_rows_beyond_32_bit_offsets(ctx):
    n, V = 14500, 151936                         # 2.2e9 logits
    z = torch.full((n, 1, V), -2.0, dtype=torch.bfloat16, device="cuda")
    hot = torch.randint(0, V, (n,), device="cuda")
    z[torch.arange(n, device="cuda"), 0, hot] = 30.0         # leaves 151935 e^-32 = 2e-9 to the others
    out = runner.verify_draft(ctx, z, None, torch.empty((n, 0), dtype=torch.int32, device="cuda"),
                              torch.empty((n, 0), device="cuda"), torch.full((n,), 0.5, device="cuda"))
    assert torch.equal(out["tokens"][:, 0].long(), hot)
    assert (out["logp"].abs() <= 6e-6).all()


def test_w4_output_beyond_32_bit_offsets(ctx):
    N, K, M, pitch = 100, 128, 20, 1 << 27       # rows of the output 2^27 elements apart: 2.5e9
    q, s, z = runner.quantize_w4(torch.randn((N, K), device="cuda"), 32)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=32)
    x = torch.randn((M, K), device="cuda").to(torch.bfloat16)
    big = torch.zeros((M - 1) * pitch + N, dtype=torch.bfloat16, device="cuda")
    out = runner.linear_w4(ctx, x, w, out=big.as_strided((M, N), (pitch, 1)))
    assert torch.equal(out, runner.linear_w4(ctx, x, w))
    assert (big[N:pitch] == 0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_an_odd_vocabulary_from_the_output_layer_to_the_verification(ctx, dtype):
    """Logits of 5003 entries in rows of 5008, as linear_w4 writes them on request; packed rows of 5003 are refused by name."""
    n_seq, N, H, V, group = 4, 2, 256, 5003, 64
    g = torch.Generator(device="cuda").manual_seed(31)
    q, s, z = runner.quantize_w4(torch.randn((V, H), generator=g, device="cuda") * 0.2, group)
    w = runner.pack_w4(ctx, q, s, z, K=H, group=group)
    h = torch.randn((n_seq * (N + 1), H), generator=g, device="cuda").to(torch.bfloat16)
    ld = (V + 7) // 8 * 8
    wide = torch.full((n_seq * (N + 1), ld), 7.0, device="cuda", dtype=dtype)
    logits = runner.linear_w4(ctx, h, w, out=wide[:, :V])
    assert logits.data_ptr() == wide.data_ptr() and (wide[:, V:] == 7).all()
    packed = runner.linear_w4(ctx, h, w, out_dtype=dtype)
    assert packed.is_contiguous() and torch.equal(packed, logits)
    target = wide.view(n_seq, N + 1, ld)[:, :, :V]
    tokens = target[:, :N].argmax(2).to(torch.int32)
    u, us = torch.rand((n_seq, N), generator=g, device="cuda") * 0.01, torch.rand(n_seq, generator=g, device="cuda")
    out = runner.verify_draft(ctx, target, None, tokens, u, us)
    logp = torch.log_softmax(target.double(), 2)
    for b in range(n_seq):
        for i in range(int(out["n_accepted"][b]) + 1):
            want = float(logp[b, i, int(out["tokens"][b, i])])
            assert abs(float(out["logp"][b, i]) - want) <= 6e-6 + U * abs(want)
    with pytest.raises(B.JackpotError, match="16 bytes"):
        runner.verify_draft(ctx, packed.view(n_seq, N + 1, V), None, tokens, u, us)
