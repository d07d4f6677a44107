"""The measured cases of the operators around the output layer: verification of drafted tokens, linear layers
with 4-bit weights, and layer norm (forward and backward).

``prepare`` makes one case's inputs from a seed, ``run`` makes one pass through an operator (its plain form in
elementary torch operations, or the framework's kernel when ``own`` is set), ``exact`` gives the same outputs
from the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "f16": torch.float16}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one user's stream: four drafted tokens against the 151,936-entry vocabulary; latency is what counts
        dict(name="verify_one_stream", op="verify", B=1, N=4, V=151936, dtype="bf16", draft="logits", ragged=False,
             temps="one", banned=False),
        # a serving step: 32 sequences with unequal numbers of drafts, some greedy, part of the vocabulary banned
        dict(name="verify_serving_step", op="verify", B=32, N=4, V=151936, dtype="bf16", draft="logits", ragged=True,
             temps="mixed", banned=True),
        # a full batch whose drafts come from a lookup of earlier text: no draft distribution, three drafts each
        dict(name="verify_lookup_drafts", op="verify", B=96, N=3, V=151936, dtype="bf16", draft="none", ragged=True,
             temps="one", banned=False),
        # fp32 logits over a vocabulary of odd width, long drafts
        dict(name="verify_f32_odd_vocab", op="verify", B=8, N=7, V=50257, dtype="f32", draft="logits", ragged=False,
             temps="mixed", banned=False),
        # one token through a square projection: the smallest call
        dict(name="w4_projection_one_token", op="w4", M=1, N=2048, K=2048, group=128, zeros=False, scales="bf16",
             out="bf16"),
        # one token through the output layer of a rollout model of hidden size 2048
        dict(name="w4_output_layer_one_token", op="w4", M=1, N=151936, K=2048, group=128, zeros=False, scales="bf16",
             out="f32"),
        # eight sequences' tokens through the output layer of a wider model, weights with zero points
        dict(name="w4_output_layer_8_tokens", op="w4", M=8, N=151936, K=4096, group=64, zeros=True, scales="f16",
             out="bf16"),
        # odd sizes, small groups, tokens of a few sequences with their drafts
        dict(name="w4_odd_19_tokens", op="w4", M=19, N=5003, K=1111, group=32, zeros=True, scales="bf16", out="f32"),
        # the norm before the output layer while decoding
        dict(name="norm_forward_decode", op="norm_fwd", T=8, H=2048, dtype="bf16", param="bf16", rms=True, bias=False),
        # a training batch's forward
        dict(name="norm_forward_train", op="norm_fwd", T=8192, H=4096, dtype="bf16", param="bf16", rms=False, bias=True),
        # fp32 activations, odd width and row count
        dict(name="norm_backward_f32_odd", op="norm_bwd", T=1531, H=1283, dtype="f32", param="f32", rms=False, bias=True),
        # a training batch's backward
        dict(name="norm_backward_train", op="norm_bwd", T=8192, H=4096, dtype="bf16", param="bf16", rms=True, bias=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["verify", "verify", "w4", "w4", "norm_fwd", "norm_bwd"])
    if op == "verify":
        budget = 96 * 4 * 151936
        N = rng.randint(1, 8)
        draft = rng.choice(["logits", "logits", "none"])
        rows = 2 * N + 1 if draft == "logits" else N + 1
        V = _log_int(rng, 1000, 200000)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        B = _log_int(rng, 1, max(1, min(128, budget // (rows * V * (1 if dtype == "bf16" else 2)))))
        return dict(op="verify", B=B, N=N, V=V, dtype=dtype, draft=draft, ragged=rng.random() < 0.5,
                    temps=rng.choice(["one", "mixed"]), banned=rng.random() < 0.5)
    if op == "w4":
        M = _log_int(rng, 1, 32)
        K = _log_int(rng, 64, 8192)
        N = _log_int(rng, 64, min(151936, 151936 * 4096 // K))
        return dict(op="w4", M=M, N=N, K=K, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5,
                    scales=rng.choice(["bf16", "f16"]), out=rng.choice(["bf16", "f32"]))
    H = _log_int(rng, 16, 8192)
    dtype = rng.choice(["bf16", "f32"])
    T = _log_int(rng, 1, min(32768, 8192 * 4096 // (H * (1 if dtype == "bf16" else 2))))
    return dict(op=op, T=T, H=H, dtype=dtype, param=rng.choice(["f32", dtype]), rms=rng.random() < 0.5,
                bias=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _verify_inputs(c, seed):
    g = _gen(seed)
    B, N, V, dt = c["B"], c["N"], c["V"], DTYPES[c["dtype"]]
    ld = (V + 7) // 8 * 8                       # rows start on 16-byte boundaries, as the output layer leaves them
    banned = torch.rand(V, device=DEV, generator=g) < 0.01 if c["banned"] else None
    target = torch.empty((B, N + 1, ld), dtype=dt, device=DEV)
    draft = torch.empty((B, N, ld), dtype=dt, device=DEV) if c["draft"] == "logits" else None
    tokens = torch.empty((B, N), dtype=torch.int32, device=DEV)
    temperature = None
    if c["temps"] == "mixed":
        pick = torch.rand(B, device=DEV, generator=g)
        temperature = torch.where(pick < 0.2, torch.zeros_like(pick), 0.5 + pick)
    for b in range(B):                          # logits of a peaked model: wide noise and a few likely tokens per row
        z = torch.randn((N + 1, V), device=DEV, generator=g) * 2.0
        spots = torch.randint(0, V, (N + 1, 6), device=DEV, generator=g)
        z.scatter_add_(1, spots, 8.0 + 6.0 * torch.rand((N + 1, 6), device=DEV, generator=g))
        zd = z[:N] + 0.5 * torch.randn((N, V), device=DEV, generator=g)      # the draft model: near the target
        if banned is not None:
            z[:, banned] = -math.inf
            zd[:, banned] = -math.inf
        target[b, :, :V] = z.to(dt)
        zd = zd.to(dt)
        if draft is not None:
            draft[b, :, :V] = zd
        t = 1.0 if temperature is None else temperature[b].clamp(min=0.05)
        noise = -torch.log(-torch.log(torch.rand((N, V), device=DEV, generator=g).clamp(1e-12, 1 - 1e-7)))
        tokens[b] = (zd.float() / t + noise).argmax(1).to(torch.int32)       # a draw from the draft model
    target[:, :, V:] = 0
    if draft is not None:
        draft[:, :, V:] = 0
    n_draft = torch.randint(0, N + 1, (B,), device=DEV, generator=g, dtype=torch.int32) if c["ragged"] else None
    return dict(target=target[:, :, :V], draft=None if draft is None else draft[:, :, :V], tokens=tokens,
                u_accept=torch.rand((B, N), device=DEV, generator=g), u_sample=torch.rand(B, device=DEV, generator=g),
                n_draft=n_draft, temperature=temperature)


def _w4_inputs(c, seed):
    g = _gen(seed)
    M, N, K, group = c["M"], c["N"], c["K"], c["group"]
    G = (K + group - 1) // group
    # two 4-bit values a byte, the lower index in the low half; sums of four draws give a bell over 0..15
    q = torch.zeros((N, (K + 1) // 2), dtype=torch.uint8, device=DEV)
    for half in (0, 1):
        parts = torch.randint(0, 2**31 - 1, (N, (K + 1) // 2), device=DEV, generator=g, dtype=torch.int32)
        v = (parts & 3) + ((parts >> 2) & 3) + ((parts >> 4) & 3) + ((parts >> 6) & 7)
        v = v.clamp_(0, 15)
        if half == 1 and K % 2:
            v[:, -1] = 0
        q |= (v << (4 * half)).to(torch.uint8)
    scales = ((0.5 + torch.rand((N, G), device=DEV, generator=g)) * (0.3 / math.sqrt(K))).to(DTYPES[c["scales"]])
    zeros = torch.randint(5, 12, (N, G), device=DEV, generator=g, dtype=torch.int32).to(torch.uint8) if c["zeros"] else None
    x = torch.randn((M, K), device=DEV, generator=g)
    x *= 1.0 + 4.0 * (torch.rand(K, device=DEV, generator=g) < 0.02)          # some hidden channels are large
    return dict(x=x.to(torch.bfloat16), q=q, scales=scales, zeros=zeros)


def _norm_inputs(c, seed):
    g = _gen(seed)
    T, H, dt, pt = c["T"], c["H"], DTYPES[c["dtype"]], DTYPES[c["param"]]
    x = torch.randn((T, H), device=DEV, generator=g) * (0.5 + torch.rand((T, 1), device=DEV, generator=g)) + 0.3
    x *= 1.0 + 9.0 * (torch.rand(H, device=DEV, generator=g) < 0.01)          # some hidden channels are large
    s = dict(x=x.to(dt), weight=(1.0 + 0.2 * torch.randn(H, device=DEV, generator=g)).to(pt),
             bias=(0.1 * torch.randn(H, device=DEV, generator=g)).to(pt) if c["bias"] else None)
    if c["op"] == "norm_bwd":                   # what a forward pass left, and the gradient that arrives
        xf = s["x"].double()
        mean = torch.zeros(T, dtype=torch.float64, device=DEV) if c["rms"] else xf.mean(1)
        var = ((xf - mean[:, None]) ** 2).mean(1)
        s["mean"] = None if c["rms"] else mean.float()
        s["rstd"] = (1.0 / torch.sqrt(var + EPS)).float()
        s["dy"] = (torch.randn((T, H), device=DEV, generator=g) / T).to(dt)
    return s


EPS = 1e-6


def _inputs(case, seed):
    if case["op"] == "verify":
        return _verify_inputs(case, seed)
    if case["op"] == "w4":
        return _w4_inputs(case, seed)
    return _norm_inputs(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = dict(case)
    if own:
        from paper_2602_06107_b200 import binding, runner
        s["ctx"] = binding.Context(torch.cuda.current_device())
        s["runner"] = runner
        if case["op"] == "w4":                  # a model's weights are laid out once, when it is loaded
            s["w"] = runner.pack_w4(s["ctx"], s["q"], s["scales"], s["zeros"], K=case["K"], group=case["group"])
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        r, ctx = state["runner"], state["ctx"]
        if op == "verify":
            o = r.verify_draft(ctx, state["target"], state["draft"], state["tokens"], state["u_accept"],
                               state["u_sample"], n_draft=state["n_draft"], temperature=state["temperature"])
            return o["n_accepted"], o["tokens"], o["accept_prob"], o["logp"]
        if op == "w4":
            return r.linear_w4(ctx, state["x"], state["w"], out_dtype=DTYPES[state["case"]["out"]])
        if op == "norm_fwd":
            return _some(r.layer_norm(ctx, state["x"], state["weight"], state["bias"], eps=EPS, rms=state["case"]["rms"]))
        return _some(r.layer_norm_backward(ctx, state["dy"], state["x"], state["weight"], state["mean"], state["rstd"],
                                           rms=state["case"]["rms"], bias=state["case"]["bias"]))
    if op == "verify":
        return _plain_verify(state)
    if op == "w4":
        return _plain_w4(state)
    if op == "norm_fwd":
        return _plain_norm_fwd(state)
    return _plain_norm_bwd(state)


def _some(outputs):
    return tuple(o for o in outputs if o is not None)


def _first_max(z):
    """Lowest index of the largest value of each row."""
    V = z.shape[-1]
    at = torch.arange(V, device=z.device)
    return torch.where(z == z.amax(-1, keepdim=True), at, V).amin(-1)


def _plain_verify(s):
    # 64 bits: a decision compares a random number with a ratio, and a draw with a sum over the vocabulary
    target, draft, tok = s["target"], s["draft"], s["tokens"].long()
    B, N1, V = target.shape
    N = N1 - 1
    temp = torch.ones(B, device=target.device) if s["temperature"] is None else s["temperature"]
    greedy = temp == 0
    t = torch.where(greedy, torch.ones_like(temp), temp).double()[:, None, None]
    n_draft = torch.full((B,), N, device=target.device) if s["n_draft"] is None else s["n_draft"].long()
    z = target.double() / t
    m = z.amax(-1, keepdim=True)
    lse = m + torch.log(torch.exp(z - m).sum(-1, keepdim=True))
    lp = z[:, :N].gather(2, tok[:, :, None])[..., 0] - lse[:, :N, 0]
    if draft is not None:
        zd = draft.double() / t
        md = zd.amax(-1, keepdim=True)
        lsed = md + torch.log(torch.exp(zd - md).sum(-1, keepdim=True))
        lq = zd.gather(2, tok[:, :, None])[..., 0] - lsed[..., 0]
    else:
        lq = torch.zeros_like(lp)
    best = _first_max(target)
    ratio = torch.where(greedy[:, None], (tok == best[:, :N]).double(), torch.exp(lp - lq))
    ok = (s["u_accept"].double() < ratio) & (torch.arange(N, device=tok.device)[None] < n_draft[:, None])
    run_ok = torch.cumprod(ok.long(), 1)
    n_acc = run_ok.sum(1)
    decided = (torch.arange(N, device=tok.device)[None] <= n_acc[:, None]) \
        & (torch.arange(N, device=tok.device)[None] < n_draft[:, None])
    accept_prob = torch.where(decided, ratio.clamp(max=1.0), torch.zeros_like(ratio)).float()

    at = torch.arange(B, device=tok.device)
    p = torch.exp(z[at, n_acc] - lse[at, n_acc])
    rejected = n_acc < n_draft
    row = n_acc.clamp(max=N - 1)
    if draft is not None:
        q = torch.exp(zd[at, row] - lsed[at, row])
    else:
        q = torch.zeros_like(p)
        q[at, tok[at, row]] = 1.0
    r = torch.where(rejected[:, None], (p - q).clamp(min=0.0), p)
    r = torch.where((r.sum(1) > 0)[:, None], r, p)
    cum = torch.cumsum(r, 1)
    want = s["u_sample"].double()[:, None] * cum[:, -1:]
    drawn = (cum <= want).sum(1).clamp(max=V - 1)
    drawn = torch.where(greedy, best[at, n_acc], drawn)
    place = torch.arange(N1, device=tok.device)[None]
    padded = torch.cat([tok, torch.zeros((B, 1), dtype=tok.dtype, device=tok.device)], 1)
    out = torch.where(place < n_acc[:, None], padded, torch.where(place == n_acc[:, None], drawn[:, None], -1))
    emitted = out.clamp(min=0)                  # log-probabilities of what was emitted: the record a rollout keeps
    logp = torch.where(out >= 0, z.gather(2, emitted[:, :, None])[..., 0] - lse[..., 0], 0.0).float()
    return n_acc.int(), out.int(), accept_prob, logp


def _plain_w4(s):
    c = s["case"]
    K, group = c["K"], c["group"]
    q = s["q"]
    v = torch.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1)[:, :K].float()
    z = 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(group, 1)[:, :K]
    w = (v - z) * s["scales"].float().repeat_interleave(group, 1)[:, :K]
    return (s["x"].float() @ w.t()).to(DTYPES[c["out"]])


def _plain_norm_fwd(s):
    c, x = s["case"], s["x"].float()
    mean = x.mean(1, keepdim=True)
    d = x if c["rms"] else x - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
    y = d * rstd * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    y = y.to(s["x"].dtype)
    return (y, rstd[:, 0]) if c["rms"] else (y, mean[:, 0], rstd[:, 0])


def _plain_norm_bwd(s):
    c, x, dy, w = s["case"], s["x"].float(), s["dy"].float(), s["weight"].float()
    rstd = s["rstd"][:, None]
    xhat = x * rstd if c["rms"] else (x - s["mean"][:, None]) * rstd
    g = dy * w
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if not c["rms"]:
        dx = dx - g.mean(1, keepdim=True)
    out = [(dx * rstd).to(s["x"].dtype), (dy * xhat).sum(0)]
    if c["bias"]:
        out.append(dy.sum(0))
    return tuple(out)


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    es = {"bf16": 2, "f16": 2, "f32": 4}
    if case["op"] == "verify":
        B, N, V = case["B"], case["N"], case["V"]
        rows = B * (N + 1) + (B * N if case["draft"] == "logits" else 0)
        if case["ragged"]:                      # half of the drafts' rows on average
            rows = B * (N / 2 + 1) + (B * N / 2 if case["draft"] == "logits" else 0)
        return {"bytes": int(rows * V * es[case["dtype"]] + B * N * 20 + B * 28), "flops": int(rows * V * 4)}
    if case["op"] == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        G = (K + case["group"] - 1) // case["group"]
        b = N * ((K + 1) // 2) + N * G * 2 + M * K * 2 + M * N * es[case["out"]]
        if case["zeros"]:
            b += N * G // 2
        return {"bytes": b, "flops": 2 * M * N * K}
    T, H, e, pe = case["T"], case["H"], es[case["dtype"]], es[case["param"]]
    if case["op"] == "norm_fwd":
        return {"bytes": 2 * T * H * e + 2 * H * pe + 8 * T, "flops": 8 * T * H}
    return {"bytes": 3 * T * H * e + H * pe + 8 * H + 8 * T, "flops": 14 * T * H}


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "verify":
        return _exact_verify(case, s)
    if case["op"] == "w4":
        return _exact_w4(case, s)
    x = s["x"].to(torch.float64)
    w = s["weight"].to(torch.float64)
    H = case["H"]
    if case["op"] == "norm_fwd":
        mu = torch.zeros(x.shape[0], dtype=torch.float64, device=DEV) if case["rms"] else x.sum(1) / H
        d = x - mu.unsqueeze(1)
        rstd = (d.pow(2).sum(1) / H + EPS).rsqrt()
        y = d * rstd.unsqueeze(1) * w
        if s["bias"] is not None:
            y = y + s["bias"].to(torch.float64)
        return (y, rstd) if case["rms"] else (y, mu, rstd)
    dy, rstd = s["dy"].to(torch.float64), s["rstd"].to(torch.float64)
    mu = torch.zeros_like(rstd) if case["rms"] else s["mean"].to(torch.float64)
    xhat = (x - mu.unsqueeze(1)) * rstd.unsqueeze(1)
    g = dy * w
    dx = g - xhat * ((g * xhat).sum(1) / H).unsqueeze(1)
    if not case["rms"]:
        dx = dx - (g.sum(1) / H).unsqueeze(1)
    out = [dx * rstd.unsqueeze(1), torch.einsum("th,th->h", dy, xhat)]
    if case["bias"]:
        out.append(torch.einsum("th->h", dy))
    return tuple(out)


def _exact_verify(case, s):
    B, N, V = case["B"], case["N"], case["V"]
    n_out = torch.zeros(B, dtype=torch.int32)
    tok_out = torch.full((B, N + 1), -1, dtype=torch.int32)
    prob_out = torch.zeros((B, N), dtype=torch.float64)
    logp_out = torch.zeros((B, N + 1), dtype=torch.float64)
    for b in range(B):
        temp = 1.0 if s["temperature"] is None else float(s["temperature"][b])
        n = N if s["n_draft"] is None else int(s["n_draft"][b])
        toks = s["tokens"][b].tolist()
        zt = s["target"][b].to(torch.float64)
        accepted = 0
        residual = None
        while accepted < n:                     # the sequential procedure, one drafted token after the other
            i, x = accepted, toks[accepted]
            if temp == 0.0:
                a = 1.0 if int((zt[i] == zt[i].max()).nonzero()[0]) == x else 0.0
            else:
                lp = torch.log_softmax(zt[i] / temp, 0)
                if s["draft"] is None:
                    lq = None
                    a = float(torch.exp(lp[x]))
                else:
                    lq = torch.log_softmax(s["draft"][b, i].to(torch.float64) / temp, 0)
                    a = float(torch.exp(lp[x] - lq[x]))
            prob_out[b, i] = min(1.0, a)
            if float(s["u_accept"][b, i]) < a:
                accepted += 1
                continue
            if temp != 0.0:
                p = lp.exp()
                if lq is None:
                    residual = p.clone()
                    residual[x] = 0.0
                else:
                    residual = (p - lq.exp()).clamp_(min=0.0)
                if float(residual.sum()) <= 0.0:
                    residual = p
            break
        n_out[b] = accepted
        tok_out[b, :accepted] = torch.tensor(toks[:accepted], dtype=torch.int32)
        if temp == 0.0:
            nxt = int((zt[accepted] == zt[accepted].max()).nonzero()[0])
        else:
            r = residual if residual is not None else torch.log_softmax(zt[accepted] / temp, 0).exp()
            c = torch.cumsum(r, 0)
            want = (float(s["u_sample"][b]) * c[-1]).reshape(1)
            nxt = min(int(torch.searchsorted(c, want, right=True)), V - 1)
        tok_out[b, accepted] = nxt
        lp = torch.log_softmax(zt / (1.0 if temp == 0.0 else temp), 1)
        for i in range(accepted + 1):
            logp_out[b, i] = lp[i, int(tok_out[b, i])]
    return n_out.to(DEV), tok_out.to(DEV), prob_out.to(DEV), logp_out.to(DEV)


def _exact_w4(case, s):
    N, K, group = case["N"], case["K"], case["group"]
    x = s["x"].to(torch.float64)
    out = torch.empty((case["M"], N), dtype=torch.float64, device=DEV)
    grp = torch.arange(K, device=DEV) // group
    for n0 in range(0, N, 8192):                # a slice of the rows at a time: the weights are large in 64 bits
        n1 = min(N, n0 + 8192)
        w = torch.empty((n1 - n0, K), dtype=torch.float64, device=DEV)
        w[:, 0::2] = (s["q"][n0:n1] & 15)[:, :(K + 1) // 2].to(torch.float64)
        w[:, 1::2] = (s["q"][n0:n1] >> 4)[:, :K // 2].to(torch.float64)
        w -= 8.0 if s["zeros"] is None else s["zeros"][n0:n1].to(torch.float64)[:, grp]
        w *= s["scales"][n0:n1].to(torch.float64)[:, grp]
        out[:, n0:n1] = x @ w.t()
    return out
