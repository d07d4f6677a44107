"""The measured cases of the operators of an update step and of a quantised model's prompt pass: the clipped policy loss and
the preference loss with their gradients, the norms around a block with gate and residual scale (forward and backward),
and linear layers in 8-bit integers.

``prepare`` makes one case's inputs from a seed, ``run`` makes one pass through an operator (its plain form in elementary
torch operations, or the framework's kernels when ``own`` is set), ``exact`` gives the same outputs from the definition
in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # a small vocabulary's update in fp32 with odd sizes: the smallest loss call, latency is what counts
        dict(name="policy_small_f32_odd", op="policy", T=61, V=5003, dtype="f32", kl=0.02, tau=1.0, weights="mean"),
        # a micro-batch of a policy update over the 151,936-entry vocabulary, padded sequences, KL to the reference model
        dict(name="policy_update", op="policy", T=4096, V=151936, dtype="bf16", kl=0.001, tau=1.0, weights="mean"),
        # a few short pairs over an odd vocabulary in fp32
        dict(name="preference_small_f32_odd", op="preference", P=3, L=40, V=20011, dtype="f32", smooth=0.1, average=True,
             ref=False),
        # a training batch of preference pairs of unequal lengths over the 151,936-entry vocabulary
        dict(name="preference_train", op="preference", P=6, L=512, V=151936, dtype="bf16", smooth=0.0, average=False,
             ref=True),
        # between two blocks while decoding: the smallest norm call
        dict(name="block_norm_forward_decode", op="block_fwd", T=8, H=2048, dtype="bf16", param="bf16", rms=True,
             post=True, bias=False, gate="none"),
        # a training batch's forward, gated
        dict(name="block_norm_forward_train", op="block_fwd", T=8192, H=4096, dtype="bf16", param="bf16", rms=True,
             post=True, bias=False, gate="channel"),
        # layer norms with bias in fp32, odd width and row count, a gate a token
        dict(name="block_norm_backward_f32_odd", op="block_bwd", T=1531, H=1283, dtype="f32", param="f32", rms=False,
             post=True, bias=True, gate="token"),
        # a training batch's backward, gated
        dict(name="block_norm_backward_train", op="block_bwd", T=8192, H=4096, dtype="bf16", param="bf16", rms=True,
             post=True, bias=False, gate="channel"),
        # one token through a square projection: the smallest linear call
        dict(name="i8_projection_one_token", op="i8", M=1, N=2048, K=2048, out="bf16"),
        # 48 sequences' tokens through the output layer of a rollout model of hidden size 2048
        dict(name="i8_output_layer_48_tokens", op="i8", M=48, N=151936, K=2048, out="f32"),
        # odd sizes: the rest of a prompt
        dict(name="i8_odd_777_tokens", op="i8", M=777, N=5003, K=1111, out="f32"),
        # a prompt pass through a wide projection
        dict(name="i8_prompt_4096_tokens", op="i8", M=4096, N=16384, K=4096, out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["policy", "preference", "block_fwd", "block_bwd", "i8", "i8"])
    if op == "policy":
        V = _log_int(rng, 1000, 200000)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        T = _log_int(rng, 1, min(65536, 4096 * 151936 // (V * (1 if dtype == "bf16" else 2))))
        return dict(op=op, T=T, V=V, dtype=dtype, kl=rng.choice([0.0, 0.001, 0.02]), tau=rng.choice([1.0, 1.0, 0.7]),
                    weights=rng.choice(["mean", "tokens"]))
    if op == "preference":
        V = _log_int(rng, 1000, 200000)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        tokens = min(65536, 4096 * 151936 // (V * (1 if dtype == "bf16" else 2)))
        P = _log_int(rng, 1, max(1, min(64, tokens // 2)))
        L = _log_int(rng, 1, max(1, tokens // (2 * P)))
        return dict(op=op, P=P, L=L, V=V, dtype=dtype, smooth=rng.choice([0.0, 0.1]), average=rng.random() < 0.5,
                    ref=rng.random() < 0.7)
    if op == "i8":
        K = _log_int(rng, 64, 16384)
        N = _log_int(rng, 64, min(151936, 151936 * 4096 // K))
        M = _log_int(rng, 1, max(1, min(8192, 4096 * 16384 * 4096 // (N * K))))
        return dict(op=op, M=M, N=N, K=K, out=rng.choice(["bf16", "f32"]))
    H = _log_int(rng, 16, 8192)
    dtype = rng.choice(["bf16", "f32"])
    T = _log_int(rng, 1, min(32768, 8192 * 4096 // (H * (1 if dtype == "bf16" else 2))))
    return dict(op=op, T=T, H=H, dtype=dtype, param=rng.choice(["f32", dtype]), rms=rng.random() < 0.6,
                post=rng.random() < 0.7, bias=rng.random() < 0.4, gate=rng.choice(["none", "channel", "token", "both"]))


# ------------------------------------------------------------------------------------------------ inputs
CLIP = (0.2, 0.28)
BETA = 0.1
SCALE = 0.7071


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _logit_rows(T, V, dtype, g, tau=1.0):
    """Rows of a peaked model, a token drawn from each, and the token's log-probability."""
    ld = (V + 7) // 8 * 8                       # rows start on 16-byte boundaries, as the output layer leaves them
    logits = torch.zeros((T, ld), dtype=dtype, device=DEV)
    tokens = torch.empty(T, dtype=torch.int32, device=DEV)
    logp = torch.empty(T, device=DEV)
    step = max(1, 80_000_000 // V)
    for t0 in range(0, T, step):
        n = min(step, T - t0)
        z = torch.randn((n, V), device=DEV, generator=g).mul_(2.0)
        spots = torch.randint(0, V, (n, 6), device=DEV, generator=g)
        z.scatter_add_(1, spots, 8.0 + 6.0 * torch.rand((n, 6), device=DEV, generator=g))
        z = z.to(dtype)
        logits[t0:t0 + n, :V] = z
        # a draw: mostly a likely entry, now and then any
        pick = torch.where(torch.rand(n, device=DEV, generator=g) < 0.9, spots[:, 0],
                           torch.randint(0, V, (n,), device=DEV, generator=g))
        tokens[t0:t0 + n] = pick.to(torch.int32)
        zf = z.float().div_(tau)
        logp[t0:t0 + n] = zf.gather(1, pick[:, None])[:, 0] - torch.logsumexp(zf, 1)
    return logits[:, :V], tokens, logp


def _policy_inputs(c, seed):
    g = _gen(seed)
    T, V = c["T"], c["V"]
    logits, tokens, logp = _logit_rows(T, V, DTYPES[c["dtype"]], g, c["tau"])
    L = max(1, T // 8)                          # eight padded sequences
    length = torch.randint((L + 1) // 2, L + 1, ((T + L - 1) // L,), device=DEV, generator=g)
    at = torch.arange(T, device=DEV)
    mask = (at % L < length[at // L]).to(torch.uint8)
    adv = torch.randn((T + L - 1) // L, device=DEV, generator=g)[at // L] + 0.1
    s = dict(logits=logits, tokens=tokens, mask=mask, advantages=adv,
             logp_old=logp + 0.15 * torch.randn(T, device=DEV, generator=g),
             logp_ref=logp + 0.3 * torch.randn(T, device=DEV, generator=g) if c["kl"] > 0 else None,
             token_weight=None)
    if c["weights"] == "tokens":                # every sequence counts the same whatever its length
        s["token_weight"] = (length.float().max() / length[at // L].float())
    return s


def _preference_inputs(c, seed):
    g = _gen(seed)
    P, L = c["P"], c["L"]
    chosen = torch.randint((L + 1) // 2, L + 1, (P,), device=DEV, generator=g)
    chosen[0] = L
    length = torch.stack([chosen, L + (L + 1) // 2 - chosen], 1).view(-1)      # a pair's lengths add up to the same
    T = P * (L + (L + 1) // 2)
    start = torch.zeros(2 * P + 1, dtype=torch.int32, device=DEV)
    start[1:] = torch.cumsum(length, 0).to(torch.int32)
    logits, tokens, logp = _logit_rows(T, c["V"], DTYPES[c["dtype"]], g)
    seq = torch.repeat_interleave(torch.arange(2 * P, device=DEV), length)
    place = torch.arange(T, device=DEV) - start[seq]
    mask = (place >= length[seq] // 4).to(torch.uint8)      # the prompt's tokens take no part
    ref = None
    if c["ref"]:
        per = (logp + 0.05 * torch.randn(T, device=DEV, generator=g)).double() * mask
        ref = torch.zeros(2 * P, dtype=torch.float64, device=DEV).index_add_(0, seq, per)
        if c["average"]:
            ref /= torch.zeros(2 * P, dtype=torch.float64, device=DEV).index_add_(0, seq, mask.double()).clamp(min=1)
        ref = ref.float()
    return dict(logits=logits, tokens=tokens, mask=mask, start=start, ref=ref)


def _norm64(x, w, b, rms):
    mean = torch.zeros(x.shape[0], dtype=torch.float64, device=DEV) if rms else x.mean(1)
    rstd = 1.0 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + EPS)
    y = (x - mean[:, None]) * rstd[:, None] * w.double()
    return (y if b is None else y + b.double()), mean, rstd


def _block_inputs(c, seed):
    g = _gen(seed)
    T, H, dt, pt = c["T"], c["H"], DTYPES[c["dtype"]], DTYPES[c["param"]]
    r = torch.randn((T, H), device=DEV, generator=g) * (1.0 + 2.0 * torch.rand((T, 1), device=DEV, generator=g))
    r *= 1.0 + 9.0 * (torch.rand(H, device=DEV, generator=g) < 0.01)          # some hidden channels are large
    x = torch.randn((T, H), device=DEV, generator=g) * 0.5 + 0.1

    def vec(scale, at):
        return (at + scale * torch.randn(H, device=DEV, generator=g)).to(pt)

    s = dict(x=x.to(dt), residual=r.to(dt), weight=vec(0.2, 1.0), bias=vec(0.1, 0.0) if c["bias"] else None,
             post_weight=vec(0.2, 1.0) if c["post"] else None,
             post_bias=vec(0.1, 0.0) if c["bias"] and c["post"] else None,
             gate=vec(0.2, 0.5) if c["gate"] in ("channel", "both") else None,
             token_gate=torch.rand(T, device=DEV, generator=g) if c["gate"] in ("token", "both") else None)
    if c["op"] == "block_bwd":                  # what a forward pass left, and the gradients that arrive
        u, s["post_mean"], s["post_rstd"] = s["x"].double(), None, None
        if c["post"]:
            u, m, k = _norm64(u, s["post_weight"], s["post_bias"], c["rms"])
            s["post_mean"], s["post_rstd"] = None if c["rms"] else m.float(), k.float()
        u = u * SCALE
        if s["gate"] is not None:
            u = u * s["gate"].double()
        if s["token_gate"] is not None:
            u = u * s["token_gate"].double()[:, None]
        s["sum"] = (s.pop("residual").double() + u).to(dt)
        _, m, k = _norm64(s["sum"].double(), s["weight"], s["bias"], c["rms"])
        s["mean"], s["rstd"] = None if c["rms"] else m.float(), k.float()
        s["dy"] = (torch.randn((T, H), device=DEV, generator=g) / T).to(dt)
        s["dsum"] = (torch.randn((T, H), device=DEV, generator=g) / T).to(dt)
    return s


def _i8_inputs(c, seed):
    g = _gen(seed)
    M, N, K = c["M"], c["N"], c["K"]
    q = torch.randn((N, K), device=DEV, generator=g).mul_(36.0).round_().clamp_(-127, 127).to(torch.int8)
    scales = (0.5 + torch.rand(N, device=DEV, generator=g)) * (0.03 / math.sqrt(K))
    x = torch.randn((M, K), device=DEV, generator=g)
    x *= 1.0 + 4.0 * (torch.rand(K, device=DEV, generator=g) < 0.02)          # some hidden channels are large
    return dict(x=x.to(torch.bfloat16), q=q, scales=scales)


def _inputs(case, seed):
    op = case["op"]
    if op == "policy":
        return _policy_inputs(case, seed)
    if op == "preference":
        return _preference_inputs(case, seed)
    if op == "i8":
        return _i8_inputs(case, seed)
    return _block_inputs(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:
        from paper_2602_06107_b200 import binding, runner
        s["ctx"] = binding.Context(torch.cuda.current_device())
        s["runner"] = runner
        if case["op"] == "i8":                  # a model's weights are laid out once, when it is loaded
            s["w"] = runner.pack_i8(s["ctx"], s["q"], s["scales"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    op = c["op"]
    if own:
        r, ctx, s = state["runner"], state["ctx"], state
        if op == "policy":
            o = r.policy_loss(ctx, s["logits"], s["tokens"], s["advantages"], s["logp_old"], logp_ref=s["logp_ref"],
                              mask=s["mask"], token_weight=s["token_weight"], eps_lo=CLIP[0], eps_hi=CLIP[1],
                              kl_coef=c["kl"], temperature=c["tau"])
            return o["loss"], o["logp"], o["kl"], o["state"], o["d_logits"]
        if op == "preference":
            o = r.preference_loss(ctx, s["logits"], s["tokens"], s["start"], ref_logp=s["ref"], mask=s["mask"], beta=BETA,
                                  label_smoothing=c["smooth"], average=c["average"])
            return o["loss"], o["margin"], o["seq_logp"], o["logp"], o["d_logits"]
        if op == "i8":
            return r.linear_i8(ctx, s["x"], s["w"], out_dtype=DTYPES[c["out"]])
        if op == "block_fwd":
            o = r.block_norm(ctx, s["x"], s["residual"], s["weight"], s["bias"], post_weight=s["post_weight"],
                             post_bias=s["post_bias"], gate=s["gate"], token_gate=s["token_gate"], scale=SCALE, eps=EPS,
                             rms=c["rms"])
            return o["sum"], o["y"], o["rstd"]
        o = r.block_norm_backward(ctx, s["dy"], s["dsum"], s["x"], s["sum"], s["weight"], s["mean"], s["rstd"],
                                  post_weight=s["post_weight"], post_bias=s["post_bias"], post_mean=s["post_mean"],
                                  post_rstd=s["post_rstd"], gate=s["gate"], token_gate=s["token_gate"], scale=SCALE,
                                  rms=c["rms"], bias=c["bias"])
        return tuple(o[k] for k in GRADS if o[k] is not None)
    if op == "policy":
        return _plain_policy(state)
    if op == "preference":
        return _plain_preference(state)
    if op == "i8":
        return _plain_i8(state)
    if op == "block_fwd":
        return _plain_block_fwd(state)
    return _plain_block_bwd(state)


GRADS = ("dx", "dresidual", "dweight", "dbias", "dpost_weight", "dpost_bias", "dgate", "dtoken_gate")


def _plain_rows(logits, tokens, tau):
    """Per row exp(z - max), its sum and the token's log-probability (a row's scalars in 64 bits: the clip is a border)."""
    z = logits.float()
    if tau != 1.0:
        z = z / tau
    m = z.amax(1, keepdim=True)
    zx = z.gather(1, tokens.long()[:, None])
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    lp = (zx.double() - m.double() - torch.log(total.double()))[:, 0]
    return e, total, lp


def _plain_gradient(e, total, tokens, coef, dtype):
    d = e * (-coef / total[:, 0])[:, None]
    d.scatter_add_(1, tokens.long()[:, None], coef[:, None])
    return d.to(dtype)


def _plain_policy(s):
    c = s["case"]
    on = s["mask"] != 0
    e, total, lp = _plain_rows(s["logits"], s["tokens"], c["tau"])
    adv = s["advantages"].double()
    r = torch.exp(lp - s["logp_old"].double())
    plain, clipped = -adv * r, -adv * r.clamp(1.0 - CLIP[0], 1.0 + CLIP[1])
    live = plain >= clipped
    per = torch.maximum(plain, clipped)
    slope = torch.where(live, plain, torch.zeros_like(plain))
    kl = torch.zeros_like(lp)
    if s["logp_ref"] is not None:
        d = s["logp_ref"].double() - lp
        kl = torch.expm1(d) - d
        slope = slope - c["kl"] * torch.expm1(d)
    weight = on.double() / on.sum()
    if s["token_weight"] is not None:
        weight = weight * s["token_weight"].double()
    loss = torch.stack([(weight * per).sum() + c["kl"] * (weight * kl).sum(), (weight * per).sum(), (weight * kl).sum()])
    coef = (weight * slope / c["tau"]).float()
    zero = torch.zeros_like(lp)
    state = torch.where(on, torch.where(live, 1, 2), 0).to(torch.uint8)
    return (loss.float(), torch.where(on, lp, zero).float(), torch.where(on, kl, zero).float(), state,
            _plain_gradient(e, total, s["tokens"], coef, s["logits"].dtype))


def _plain_preference(s):
    c = s["case"]
    P, T = c["P"], s["tokens"].shape[0]
    on = s["mask"] != 0
    e, total, lp = _plain_rows(s["logits"], s["tokens"], 1.0)
    lp = torch.where(on, lp, torch.zeros_like(lp))
    seq = torch.searchsorted(s["start"].long(), torch.arange(T, device=lp.device), right=True) - 1
    sums = torch.zeros(2 * P, dtype=torch.float64, device=lp.device).index_add_(0, seq, lp)
    per = torch.ones_like(sums)
    if c["average"]:
        per = 1.0 / torch.zeros_like(sums).index_add_(0, seq, on.double()).clamp(min=1)
    sums = sums * per
    gap = (sums if s["ref"] is None else sums - s["ref"].double()).view(P, 2)
    h = BETA * (gap[:, 0] - gap[:, 1])
    up = torch.log1p(torch.exp(-h.abs()))
    loss = ((1.0 - c["smooth"]) * (up + (-h).clamp(min=0)) + c["smooth"] * (up + h.clamp(min=0))).mean()
    sig = 1.0 / (1.0 + torch.exp(-h))
    slope = (BETA / P) * (c["smooth"] * sig - (1.0 - c["smooth"]) * (1.0 - sig))
    coef = (torch.stack([slope, -slope], 1).view(-1) * per)[seq] * on
    return (loss.float().reshape(1), h.float(), sums.float(), lp.float(),
            _plain_gradient(e, total, s["tokens"], coef.float(), s["logits"].dtype))


def _plain_i8(s):
    x = s["x"].float()
    most = x.abs().amax(1, keepdim=True)
    # (64 bits: which integer is nearest)
    q = torch.where(most > 0, 127.0 * x.double() / most.double(), torch.zeros_like(x, dtype=torch.float64)).round().float()
    return (q @ s["q"].float().t() * (most / 127.0) * s["scales"]).to(DTYPES[s["case"]["out"]])


def _plain_norm(x, w, b, rms):
    mean = x.mean(1, keepdim=True)
    d = x if rms else x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    y = d * rstd * w.float()
    return (y if b is None else y + b.float()), rstd


def _plain_block_fwd(s):
    c = s["case"]
    u = s["x"].float()
    if s["post_weight"] is not None:
        u, _ = _plain_norm(u, s["post_weight"], s["post_bias"], c["rms"])
    u = u * SCALE
    if s["gate"] is not None:
        u = u * s["gate"].float()
    if s["token_gate"] is not None:
        u = u * s["token_gate"][:, None]
    total = (s["residual"].float() + u).to(s["x"].dtype)
    y, rstd = _plain_norm(total.float(), s["weight"], s["bias"], c["rms"])
    return total, y.to(s["x"].dtype), rstd[:, 0]


def _plain_norm_bwd(dy, x, w, mean, rstd, rms):
    """(dx, dy xhat): the gradient with respect to x, and what the weight's gradient sums."""
    xhat = (x if rms else x - mean[:, None]) * rstd[:, None]
    g = dy * w.float()
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if not rms:
        dx = dx - g.mean(1, keepdim=True)
    return dx * rstd[:, None], dy * xhat, xhat


def _plain_block_bwd(s):
    c, dt = s["case"], s["x"].dtype
    dy, x = s["dy"].float(), s["x"].float()
    ds, per_w, _ = _plain_norm_bwd(dy, s["sum"].float(), s["weight"], s["mean"], s["rstd"], c["rms"])
    ds = ds + s["dsum"].float()
    out = dict.fromkeys(GRADS)
    out["dresidual"], out["dweight"] = ds.to(dt), per_w.sum(0)
    if c["bias"]:
        out["dbias"] = dy.sum(0)
    u = x
    if s["post_weight"] is not None:
        xhat = (x if c["rms"] else x - s["post_mean"][:, None]) * s["post_rstd"][:, None]
        u = xhat * s["post_weight"].float()
        if s["post_bias"] is not None:
            u = u + s["post_bias"].float()
    gc = 1.0 if s["gate"] is None else s["gate"].float()
    gt = 1.0 if s["token_gate"] is None else s["token_gate"][:, None]
    if s["gate"] is not None:
        out["dgate"] = (u * ds * gt).sum(0) * SCALE
    if s["token_gate"] is not None:
        out["dtoken_gate"] = (u * ds * gc).sum(1) * SCALE
    du = ds * SCALE * gc * gt
    if s["post_weight"] is not None:
        dx, per_w, _ = _plain_norm_bwd(du, x, s["post_weight"], s["post_mean"], s["post_rstd"], c["rms"])
        out["dpost_weight"] = per_w.sum(0)
        if c["bias"]:
            out["dpost_bias"] = du.sum(0)
        du = dx
    out["dx"] = du.to(dt)
    return tuple(out[k] for k in GRADS if out[k] is not None)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    es = {"bf16": 2, "f32": 4}
    op = case["op"]
    if op == "policy":                          # valid rows (about three quarters) read, all rows of the gradient written
        T, V, e = case["T"], case["V"], es[case["dtype"]]
        return {"bytes": int((0.77 * T + T) * V * e + 30 * T), "flops": int(0.77 * T * V * 6)}
    if op == "preference":                      # rows with a part (three quarters) read twice: the scalars need whole pairs
        T, V, e = case["P"] * (case["L"] + (case["L"] + 1) // 2), case["V"], es[case["dtype"]]
        return {"bytes": int((2 * 0.75 * T + T) * V * e + 20 * T), "flops": int(0.75 * T * V * 6)}
    if op == "i8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": N * K + 4 * N + 2 * M * K + M * N * es[case["out"]], "flops": 2 * M * N * K}
    T, H, e, pe = case["T"], case["H"], es[case["dtype"]], es[case["param"]]
    if op == "block_fwd":
        return {"bytes": 4 * T * H * e + 4 * H * pe + 8 * T, "flops": 16 * T * H}
    return {"bytes": 6 * T * H * e + 4 * H * (pe + 4) + 12 * T, "flops": 36 * T * H}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("policy", "preference"):
        return _exact_loss(case, s)
    if op == "i8":
        return _exact_i8(case, s)
    return _exact_block(case, s)


def _exact_loss(case, s):
    T, V = s["logits"].shape
    tau = case.get("tau", 1.0)
    logp = torch.zeros(T, dtype=torch.float64, device=DEV)
    d_logits = torch.zeros((T, V), dtype=torch.float64, device=DEV)
    step = max(1, 20_000_000 // V)
    for t0 in range(0, T, step):                # a slice of the rows at a time: the logits are large in 64 bits
        ls = torch.log_softmax(s["logits"][t0:t0 + step].to(torch.float64) / tau, 1)
        tok = s["tokens"][t0:t0 + step].long()
        logp[t0:t0 + step] = ls[torch.arange(ls.shape[0], device=DEV), tok]
        d_logits[t0:t0 + step] = ls.exp_().neg_()
        d_logits[torch.arange(t0, t0 + ls.shape[0], device=DEV), tok] += 1.0
    valid = s["mask"].bool()
    logp = logp * valid
    free = logp.clone().requires_grad_(True)    # the loss as a function of the log-probabilities
    if case["op"] == "policy":
        ratio = (free - s["logp_old"].to(torch.float64)).exp()
        adv = s["advantages"].to(torch.float64)
        lo, hi = 1.0 - CLIP[0], 1.0 + CLIP[1]
        inside = torch.where(adv >= 0, ratio <= hi, ratio >= lo)
        bound = torch.where(adv >= 0, torch.full_like(adv, hi), torch.full_like(adv, lo))
        term = -adv * torch.where(inside, ratio, bound)
        kl = torch.zeros_like(logp)
        if s["logp_ref"] is not None:
            gap = s["logp_ref"].to(torch.float64) - free
            kl = torch.expm1(gap) - gap
        w = valid.to(torch.float64) / int(valid.sum())
        if s["token_weight"] is not None:
            w = w * s["token_weight"].to(torch.float64)
        first, second = torch.dot(w, term), torch.dot(w, kl)
        total = first + case["kl"] * second
        total.backward()
        state = (valid.to(torch.uint8) * (2 - inside.to(torch.uint8)))
        head = (torch.stack([total, first, second]).detach(), logp, (kl * valid).detach(), state)
        d_logits *= (free.grad / tau)[:, None]
        return head + (d_logits,)
    bounds = s["start"].tolist()
    sums = []
    for a, b in zip(bounds[:-1], bounds[1:]):
        part = free[a:b][valid[a:b]]
        sums.append(part.mean() if case["average"] and part.numel() else part.sum())
    sums = torch.stack(sums)
    gap = sums if s["ref"] is None else sums - s["ref"].to(torch.float64)
    h = BETA * (gap[0::2] - gap[1::2])
    ls = torch.nn.functional.logsigmoid
    loss = -((1.0 - case["smooth"]) * ls(h) + case["smooth"] * ls(-h)).mean()
    loss.backward()
    grad = torch.where(valid, free.grad, torch.zeros_like(logp))
    d_logits *= grad[:, None]
    return loss.detach().reshape(1), h.detach(), sums.detach(), logp, d_logits


def _exact_i8(case, s):
    x = s["x"].to(torch.float64)
    most = x.abs().max(1).values
    step = torch.where(most > 0, most, torch.ones_like(most))
    q = torch.round(x * 127.0 / step.unsqueeze(1))
    out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=DEV)
    for n0 in range(0, case["N"], 8192):        # a slice of the rows at a time: the weights are large in 64 bits
        w = s["q"][n0:n0 + 8192].to(torch.float64) * s["scales"][n0:n0 + 8192].to(torch.float64).unsqueeze(1)
        out[:, n0:n0 + 8192] = (q @ w.t()) * (most / 127.0).unsqueeze(1)
    return out


def _exact_block(case, s):
    def wide(t, grad=False):
        return None if t is None else t.to(torch.float64).requires_grad_(grad)

    back = case["op"] == "block_bwd"
    x, w, b = wide(s["x"], back), wide(s["weight"], back), wide(s["bias"], back)
    pw, pb, gate, tg = (wide(s[k], back) for k in ("post_weight", "post_bias", "gate", "token_gate"))

    def normed(v, weight, bias, mean=None, rstd=None):
        """The norm of each row; where the statistics are given they stand in the place of the row's own values only."""
        mu = torch.zeros_like(v[:, :1]) if case["rms"] else v.mean(1, keepdim=True)
        k = ((v - mu).pow(2).mean(1, keepdim=True) + EPS).rsqrt()
        if mean is not None:
            mu = mu + (mean.to(torch.float64)[:, None] - mu).detach()
        if rstd is not None:
            k = k + (rstd.to(torch.float64)[:, None] - k).detach()
        out = (v - mu) * k * weight
        return (out if bias is None else out + bias), k

    u = x
    if pw is not None:
        u, _ = normed(x, pw, pb, s.get("post_mean"), s.get("post_rstd"))
    u = u * SCALE
    if gate is not None:
        u = u * gate
    if tg is not None:
        u = u * tg.unsqueeze(1)
    if not back:
        # the sum is stored before its norm is taken: what is normed is what was stored
        total = s["residual"].to(torch.float64) + u
        y, k = normed(total.to(s["x"].dtype).to(torch.float64), w, b)
        return total, y, k[:, 0]
    total = wide(s["sum"], True)
    y, _ = normed(total, w, b, s["mean"], s["rstd"])
    leaves = [t for t in (w, b) if t is not None]
    got = dict(zip(["total", "w", "b"], torch.autograd.grad(y, [total] + leaves, s["dy"].to(torch.float64))))
    ds = got["total"] + s["dsum"].to(torch.float64)
    named = {"x": x, "pw": pw, "pb": pb, "gate": gate, "tg": tg}
    named = {k: v for k, v in named.items() if v is not None}
    got.update(zip(named, torch.autograd.grad(u, list(named.values()), ds)))
    out = (got["x"], ds, got["w"], got.get("b"), got.get("pw"), got.get("pb"), got.get("gate"), got.get("tg"))
    return tuple(t for t in out if t is not None)
