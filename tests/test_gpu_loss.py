"""The policy and preference losses (jp_policy_loss, jp_preference_loss) against a plain implementation in 64 bits.

Bars.  u = 2^-24, X = 2^-22: the bound on a hardware 2^x.  A row's sum: each term errs by X and by the rounding of its exponent, which weighs at
most u; a thread adds at most 300 terms (u of the sum so far each, so 150 u for terms of one distribution), and each of at most 15 merges
multiplies one side by a 2^x: below 16 X + 160 u = 56 X in all.  log takes the relative error as it is, so a log-probability errs by
E = 56 X = 1.34e-5 plus 1.34e-8 times the row's entropy (log2(e) in fp32), below 13: E = 1.36e-5, plus u of itself when it is stored.
The scalars are fp64, so ratios err by E relative, exp(d) - d - 1 by |exp(d) - 1| E, a coefficient by the derivative of its formula, and a
probability by E + 2 X relative; the gradient is rounded once more, half a step of its type."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -24, 1.36e-5
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def make(T, V, dtype, seed, pitch=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = pitch or (V + 7) // 8 * 8
    z = torch.full((T, ld), float("nan"), device="cuda", dtype=dtype)
    z[:, :V] = (torch.randn((T, V), generator=g, device="cuda") * 2).to(dtype)
    z = z[:, :V]
    if V > 8:
        spots = torch.randint(0, V, (T, 3), generator=g, device="cuda")
        z.scatter_(1, spots, (8 + 4 * torch.rand((T, 3), generator=g, device="cuda")).to(dtype))
        tok = torch.where(torch.rand(T, generator=g, device="cuda") < 0.8, spots[:, 0], torch.randint(0, V, (T,), generator=g, device="cuda"))
    else:
        tok = torch.randint(0, V, (T,), generator=g, device="cuda")
    lp = torch.log_softmax(z.double(), 1).gather(1, tok[:, None])[:, 0]
    old = (lp + 0.2 * torch.randn(T, generator=g, device="cuda", dtype=torch.float64)).float()
    ref = (lp + 0.4 * torch.randn(T, generator=g, device="cuda", dtype=torch.float64)).float()
    adv = torch.randn(T, generator=g, device="cuda")
    mask = (torch.rand(T, generator=g, device="cuda") < 0.8).to(torch.uint8)
    weight = torch.rand(T, generator=g, device="cuda") + 0.5
    return z, tok.int(), adv, old, ref, mask, weight


def as_given(*values):
    """The entries take their numbers in fp32."""
    return [float(torch.tensor(v, dtype=F32)) for v in values]


def plain_policy(z, tok, adv, old, ref, mask, weight, n_valid, lo, hi, kl_coef, tau, g):
    """Everything in 64 bits, with the sizes of what may err."""
    lo, hi, kl_coef, tau, g = as_given(lo, hi, kl_coef, tau, g)
    T = z.shape[0]
    ls = torch.log_softmax(z.double() / tau, 1)
    p = ls.exp()
    hot = torch.zeros_like(p).scatter_(1, tok.long()[:, None], 1.0)
    lp = ls.gather(1, tok.long()[:, None])[:, 0]
    on = torch.ones(T, dtype=torch.bool, device="cuda") if mask is None else mask != 0
    r = (lp - old.double()).exp()
    a = adv.double()
    plain, clipped = -a * r, -a * r.clamp(1 - lo, 1 + hi)
    live = plain >= clipped if lo or hi else torch.ones_like(on)
    loss = torch.where(live, plain, clipped)
    kl, e1 = torch.zeros_like(lp), torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        e1 = torch.expm1(d)
        kl = e1 - d
    N = n_valid or max(1, int(on.sum()))
    c = (torch.ones_like(lp) if weight is None else weight.double()) * on / N
    k = c * (torch.where(live, plain, 0.0) - kl_coef * e1) * g / tau
    k_err = c * (torch.where(live, plain.abs(), 0.0) + abs(kl_coef) * (1 + e1)) * abs(g) / tau * E
    near = ((r / (1 - lo) - 1).abs() < 4 * E) | ((r / (1 + hi) - 1).abs() < 4 * E) if lo or hi else torch.zeros_like(on)
    return dict(on=on, lp=lp, kl=kl, e1=e1, live=live, near=near & on, term=c * loss, kterm=c * kl, r=r, a=a, c=c, k=k, k_err=k_err, p=p, hot=hot)


def check_gradient(d, P, dtype, rows):
    ref = P["k"][:, None] * (P["hot"] - P["p"])
    mag = P["hot"] + P["p"]
    bar = HALF[dtype] * ref.abs() * (1 + 2.0 ** -8) + P["k_err"][:, None] * mag + P["k"].abs()[:, None] * (P["p"] * (E + 3 * 2.0 ** -22) + 2 * U * mag)
    if dtype is BF:
        bar += 1e-40
    assert (((d.double() - ref).abs() <= bar) | ~rows[:, None]).all()


def check_policy(o, dtype, P, kl_coef, grad=True):
    on = P["on"]
    assert ((o["logp"].double() - P["lp"]).abs()[on] <= E + U * P["lp"].abs()[on]).all()
    assert (o["logp"][~on] == 0).all() and (o["kl"][~on] == 0).all() and (o["state"][~on] == 0).all()
    assert ((o["kl"].double() - P["kl"]).abs()[on] <= (P["e1"].abs() * E + E * E + 2 * U * P["kl"] + 1e-12)[on]).all()
    want = torch.where(on, torch.where(P["live"], 1, 2), 0)
    assert ((o["state"].long() == want) | P["near"]).all()
    # a term on either branch near the clip differs by 4 E |A| c at most
    err = (P["c"] * P["a"].abs() * P["r"] * 4 * E).sum()
    kerr = (P["c"] * (P["e1"].abs() * E + E * E)).sum()
    s1, s2 = P["term"].sum(), P["kterm"].sum()
    for got, want, bar in zip(o["loss"].double(), (s1 + kl_coef * s2, s1, s2), (err + abs(kl_coef) * kerr, err, kerr)):
        assert (got - want).abs() <= bar + U * want.abs() + 1e-30
    if grad:
        check_gradient(o["d_logits"], P, dtype, ~P["near"])
        assert (o["d_logits"][~on] == 0).all()


SHAPES = [(1, 1), (1, 7), (3, 8), (2, 9), (5, 5003), (61, 20011), (2, 151936), (40, 151936), (700, 1000), (300, 32000), (1, 600001), (160, 131072)]


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form", ["all", "bare"])
def test_policy_matches_the_formula(ctx, T, V, dtype, form):
    z, tok, adv, old, ref, mask, weight = make(T, V, dtype, T + V)
    if form == "all":
        args = dict(logp_ref=ref, mask=mask, token_weight=weight, n_valid=3, eps_lo=0.2, eps_hi=0.28, kl_coef=0.05, temperature=0.7, grad_out=2.0)
        old = old + (torch.log_softmax(z.double() / 0.7, 1) - torch.log_softmax(z.double(), 1)).gather(1, tok.long()[:, None])[:, 0].float()
        P = plain_policy(z, tok, adv, old, ref, mask, weight, 3, 0.2, 0.28, 0.05, 0.7, 2.0)
    else:
        args = dict(eps_lo=0.0, eps_hi=0.0)
        P = plain_policy(z, tok, adv, old, None, None, None, 0, 0.0, 0.0, 0.0, 1.0, 1.0)
    keep = z.clone()
    o = runner.policy_loss(ctx, z, tok, adv, old, **args)
    check_policy(o, dtype, P, args.get("kl_coef", 0.0))
    assert torch.equal(z, keep) or z.isnan().any()
    again = runner.policy_loss(ctx, z, tok, adv, old, **args)
    assert all(torch.equal(again[k], o[k]) for k in o)
    without = runner.policy_loss(ctx, z, tok, adv, old, grad=False, **args)
    assert without["d_logits"] is None                       # (another order of sums)
    check_policy(without, dtype, P, args.get("kl_coef", 0.0), grad=False)
    inside = runner.policy_loss(ctx, z, tok, adv, old, d_logits=z, **args)             # the gradient in the logits' place
    assert inside["d_logits"].data_ptr() == z.data_ptr() and torch.equal(z, o["d_logits"]) and torch.equal(inside["loss"], o["loss"])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_policy_counts_its_rows(ctx, dtype):
    """N from the mask, wherever the mask starts; the mean of a constant is the constant."""
    for T, off in ((1, 0), (31, 1), (700, 3), (4099, 15), (2048, 0)):
        z, tok, adv, old, ref, mask, weight = make(T, 40, dtype, T)
        m = torch.zeros(T + off, dtype=torch.uint8, device="cuda")[off:]
        m.copy_(mask * 255)
        m[0] = 1
        o = runner.policy_loss(ctx, z, tok, torch.ones_like(adv), old, mask=m, eps_lo=0.1, eps_hi=0.1)
        P = plain_policy(z, tok, torch.ones_like(adv), old, None, m, None, 0, 0.1, 0.1, 0.0, 1.0, 1.0)
        check_policy(o, dtype, P, 0.0)


def test_masked_throughout_and_no_rows(ctx):
    z, tok, adv, old, ref, mask, weight = make(9, 100, F32, 1)
    o = runner.policy_loss(ctx, z, tok, adv, old, logp_ref=ref, mask=torch.zeros_like(mask), kl_coef=0.1)
    assert (o["loss"] == 0).all() and (o["d_logits"] == 0).all() and (o["state"] == 0).all()
    o = runner.policy_loss(ctx, z[:0], tok[:0], adv[:0], old[:0])
    assert (o["loss"] == 0).all() and o["d_logits"].shape == (0, 100)
    start = torch.zeros(1, dtype=torch.int32, device="cuda")
    o = runner.preference_loss(ctx, z[:0], tok[:0], start)
    assert (o["loss"] == 0).all() and o["d_logits"].shape == (0, 100) and o["margin"].numel() == 0
    o = runner.preference_loss(ctx, z, tok, start)                                     # rows, but no pairs
    assert (o["loss"] == 0).all() and (o["d_logits"] == 0).all() and (o["state"] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_policy_rows_without_numbers(ctx, dtype):
    """Such rows take no part and the others do not change."""
    T, V = 24, 5000
    z, tok, adv, old, ref, _, weight = make(T, V, dtype, 5)
    low = float(torch.finfo(dtype).min)
    z[1, 17] = float("nan")
    z[2, 4999] = float("inf")
    z[3, :] = float("-inf")
    z[4, :] = low
    tok[5], tok[6] = -1, V
    tok[7] = 11
    z[7, 11] = float("-inf")                     # the token has probability 0
    old[8] = float("nan")
    adv[9] = float("inf")
    ref[10] = float("inf")
    bad = [1, 2, 3, 4, 7, 8, 9, 10]
    z[11, ::2] = float("-inf")                   # entries without probability, by either way of masking
    z[12, ::2] = low
    for i in (11, 12):
        tok[i] = 2 * (int(tok[i]) // 2) + 1
        old[i] = ref[i] = torch.log_softmax(z[i].double(), 0)[tok[i].long()].float() - 0.05
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    o = runner.policy_loss(ctx, z, tok, adv, old, logp_ref=ref, mask=mask, token_weight=weight, n_valid=T, kl_coef=0.1)
    assert (o["state"][bad] == 3).all() and (o["state"][[5, 6]] == 0).all()
    out = bad + [5, 6]
    assert (o["d_logits"][out] == 0).all() and (o["logp"][out] == 0).all() and (o["kl"][out] == 0).all()
    good = [i for i in range(T) if i not in out]
    sub = lambda t: t[good].contiguous()
    P = plain_policy(z[good], sub(tok), sub(adv), sub(old), sub(ref), None, sub(weight), T, 0.2, 0.2, 0.1, 1.0, 1.0)
    check_policy({k: (v if k == "loss" else v[good]) for k, v in o.items()}, dtype, P, 0.1)
    assert (o["d_logits"][11, ::2] == 0).all() and (o["d_logits"][12, ::2] == 0).all()
    # without a KL term a token of probability 0 is a row like others: ratio 0
    o = runner.policy_loss(ctx, z, tok, adv, old, mask=mask)
    assert o["state"][7] in (1, 2) and o["logp"][7] == float("-inf") and (o["d_logits"][7] == 0).all() and o["loss"].isfinite().all()


def test_gradients_against_differences(ctx):
    T, V, h = 5, 23, 1e-5
    z, tok, adv, old, ref, _, weight = make(T, V, F32, 3)
    mask = torch.tensor([1, 1, 0, 1, 1], dtype=torch.uint8, device="cuda")
    o = runner.policy_loss(ctx, z, tok, adv, old, logp_ref=ref, mask=mask, token_weight=weight, kl_coef=0.3, temperature=1.3)
    start = torch.tensor([0, 2, 5], dtype=torch.int32, device="cuda")
    q = runner.preference_loss(ctx, z, tok, start, mask=mask, beta=0.5, label_smoothing=0.2, margin=0.1)

    def policy(zz):
        P = plain_policy(zz, tok, adv, old, ref, mask, weight, 0, 0.2, 0.2, 0.3, 1.3, 1.0)
        return float(P["term"].sum() + 0.3 * P["kterm"].sum())

    def pref(zz):
        return float(plain_preference(zz, tok, start, None, mask, 0.5, 0.2, 0.1, False, 1.0)["loss"])
    for f, d in ((policy, o["d_logits"]), (pref, q["d_logits"])):
        for i in range(0, T * V, 3):
            up, down = z.double().clone(), z.double().clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            # h^2 times a third derivative of order 10, and 2^-52 |loss| / h: below 1e-8; the gradient errs by E and u of at most 3
            assert abs((f(up) - f(down)) / (2 * h) - float(d.reshape(-1)[i])) <= 5 * E


def plain_preference(z, tok, start, ref, mask, beta, eps, margin, average, g):
    beta, eps, margin, g = as_given(beta, eps, margin, g)
    ls = torch.log_softmax(z.double(), 1)
    T = z.shape[0]
    n = start.numel() - 1
    lp = ls.gather(1, tok.long().clamp(0, z.shape[1] - 1)[:, None])[:, 0]
    at = torch.arange(T, device="cuda")
    on = (at >= start[0]) & (at < start[-1])
    if mask is not None:
        on &= mask != 0
    seq = (torch.searchsorted(start.long(), at, right=True) - 1).clamp(0, max(n - 1, 0))
    used = torch.where(on, lp, 0.0)
    S, C = (torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, seq, v) for v in (used, on.double()))
    per = 1 / C.clamp(min=1) if average else torch.ones_like(C)
    S, C = S * per, C * per
    gap = S if ref is None else S - ref.double()
    h = beta * (gap[0::2] - gap[1::2]) - margin
    sp = torch.nn.functional.softplus
    loss = ((1 - eps) * sp(-h) + eps * sp(h))
    slope = beta * g / (n // 2) * (eps * torch.sigmoid(h) - (1 - eps) * torch.sigmoid(-h))
    k = (torch.stack([slope, -slope], 1).view(-1) * per)[seq] * on
    # h errs by beta E a valid row (its mean with average), the slope by beta / P of a quarter of that
    h_err = abs(beta) * E * (C[0::2] + C[1::2])
    s_err = abs(beta * g) / (n // 2) * h_err / 4
    k_err = (torch.stack([s_err, s_err], 1).view(-1) * per)[seq] * on
    hot = torch.zeros_like(ls).scatter_(1, tok.long()[:, None], 1.0)
    return dict(on=on, lp=lp, S=S, C=C, h=h, h_err=h_err, loss=loss.mean(), k=k, k_err=k_err, p=ls.exp(), hot=hot)


def check_preference(o, dtype, P, grad=True):
    on = P["on"]
    assert ((o["logp"].double() - P["lp"]).abs()[on] <= E + U * P["lp"].abs()[on]).all()
    assert (o["logp"][~on] == 0).all() and torch.equal(o["state"].bool(), on)
    assert ((o["seq_logp"].double() - P["S"]).abs() <= E * P["C"] + U * P["S"].abs()).all()
    assert ((o["margin"].double() - P["h"]).abs() <= P["h_err"] + 2 * U * P["h"].abs()).all()
    assert (o["loss"].double() - P["loss"]).abs() <= P["h_err"].mean() + U * P["loss"].abs() + 1e-30
    if grad:
        check_gradient(o["d_logits"], P, dtype, torch.ones_like(on))
        assert (o["d_logits"][~on] == 0).all()


def lengths_of(P, most, seed):
    g = torch.Generator().manual_seed(seed)
    n = torch.randint(0, most + 1, (2 * P,), generator=g)
    n[0] = most
    return n


@pytest.mark.parametrize("P,most,V", [(1, 1, 5), (1, 3, 20011), (4, 9, 151936), (300, 3, 257), (3, 70, 5003), (2, 60, 131072), (700, 2, 64)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("average,eps", [(False, 0.0), (True, 0.1)])
def test_preference_matches_the_formula(ctx, P, most, V, dtype, average, eps):
    """Sequences of any length, none among them, with rows in front of the first and behind the last."""
    n = lengths_of(P, most, P + V)
    front, behind = (2, 3) if average else (0, 0)
    start = (torch.cat([torch.zeros(1, dtype=torch.int64), n.cumsum(0)]) + front).int().cuda()
    T = int(n.sum()) + front + behind
    z, tok, _, _, _, mask, _ = make(T, V, dtype, P + most + V)
    g = torch.Generator(device="cuda").manual_seed(1)
    ref = None if average and P == 1 else torch.randn(2 * P, generator=g, device="cuda") * 2 - 2
    args = dict(ref_logp=ref, mask=mask if eps else None, beta=0.3, label_smoothing=eps, margin=0.2 if average else 0.0, average=average,
                grad_out=1.5)
    o = runner.preference_loss(ctx, z, tok, start, **args)
    R = plain_preference(z, tok, start, ref, args["mask"], 0.3, eps, args["margin"], average, 1.5)
    check_preference(o, dtype, R)
    again = runner.preference_loss(ctx, z, tok, start, **args)
    assert all(torch.equal(again[k], o[k]) for k in o)
    without = runner.preference_loss(ctx, z, tok, start, grad=False, **args)
    assert without["d_logits"] is None and all(torch.equal(without[k], o[k]) for k in ("loss", "logp", "margin", "seq_logp", "state"))
    inside = runner.preference_loss(ctx, z, tok, start, d_logits=z, **args)
    assert torch.equal(z, o["d_logits"]) and torch.equal(inside["loss"], o["loss"])


@pytest.mark.parametrize("V", [5, 513, 1030, 2049, 4100, 7167, 7180, 8200])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_short_rows(ctx, V, dtype):
    """More rows than four an SM, by length."""
    for form in ("all", "bare"):
        test_policy_matches_the_formula(ctx, 1311, V, dtype, form)
    for average, eps in ((False, 0.0), (True, 0.1)):
        test_preference_matches_the_formula(ctx, 40, 60, V, dtype, average, eps)


def test_preference_far_apart_and_without_numbers(ctx):
    """Pairs far apart on either side keep the small sigma; a row without numbers leaves its sequence's others."""
    T, V = 8, 300
    z, tok, _, _, _, _, _ = make(T, V, F32, 8)
    start = torch.tensor([0, 2, 4, 6, 8], dtype=torch.int32, device="cuda")
    ref = torch.tensor([-400.0, 0.0, 400.0, 0.0], device="cuda")
    o = runner.preference_loss(ctx, z, tok, start, ref_logp=ref, beta=0.2)
    check_preference(o, F32, plain_preference(z, tok, start, ref, None, 0.2, 0.0, 0.0, False, 1.0))
    assert (o["d_logits"][:4] != 0).any()                                               # 1 - sigma(80), about 1e-35
    z[1, 5] = float("nan")
    tok[6] = -3
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    o = runner.preference_loss(ctx, z, tok, start, beta=0.2, average=True)
    assert o["state"].tolist() == [1, 3, 1, 1, 1, 1, 0, 1]
    mask[1] = mask[6] = 0
    z[1, 5], tok[6] = 0.0, 0
    R = plain_preference(z, tok, start, None, mask, 0.2, 0.0, 0.0, True, 1.0)
    check_preference({**o, "state": o["state"] % 3}, F32, R)


def test_preference_without_pairs_and_with_a_reference_that_is_no_number(ctx):
    z, tok, _, _, _, _, _ = make(6, 300, F32, 9)
    o = runner.preference_loss(ctx, z, tok, torch.tensor([2], dtype=torch.int32, device="cuda"))
    assert o["loss"].item() == 0 and (o["d_logits"] == 0).all() and (o["state"] == 0).all() and o["margin"].numel() == 0
    start = torch.tensor([0, 1, 3, 4, 6], dtype=torch.int32, device="cuda")
    ref = torch.tensor([float("nan"), 0.0, -3.0, -4.0], device="cuda")
    o = runner.preference_loss(ctx, z, tok, start, ref_logp=ref)
    clean = runner.preference_loss(ctx, z, tok, start, ref_logp=torch.nan_to_num(ref))
    assert o["loss"].isnan() and o["margin"][0].isnan() and o["margin"][1] == clean["margin"][1]
    assert (o["d_logits"][:3] == 0).all() and torch.equal(o["d_logits"][3:], clean["d_logits"][3:])


def test_offsets_beyond_32_bits(ctx):
    """4500 rows of 500,000 bf16: more than 2^31 elements, 4.5 GB; the last row is the first one's copy."""
    T, V = 4500, 500000
    z = torch.zeros((T, V), device="cuda", dtype=BF)
    row, tok1, adv1, old1, ref1, _, _ = make(1, V, BF, 2)
    z[0] = z[T - 1] = row[0]
    tok = torch.zeros(T, dtype=torch.int32, device="cuda")
    tok[0] = tok[T - 1] = tok1[0]
    adv, old = torch.ones(T, device="cuda"), torch.zeros(T, device="cuda")
    old[0] = old[T - 1] = old1[0]
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    mask[0] = mask[T - 1] = 1
    # (without clipping: the gradient of a clipped row is 0 throughout)
    o = runner.policy_loss(ctx, z, tok, adv, old, mask=mask, eps_lo=0.0, eps_hi=0.0)
    assert torch.equal(o["d_logits"][0], o["d_logits"][T - 1]) and (o["d_logits"][0] != 0).any()
    assert (o["d_logits"][1:T - 1:97] == 0).all()
    P = plain_policy(row, tok1, adv[:1], old1, None, None, None, 2, 0.0, 0.0, 0.0, 1.0, 1.0)
    check_gradient(o["d_logits"][:1], P, BF, ~P["near"])


def test_streams_graphs_and_workspaces(ctx):
    """Two streams at once, and two captured graphs that are replayed with new inputs."""
    a = make(300, 20000, BF, 1)
    b = make(300, 20000, BF, 2)
    start = torch.tensor([0, 100, 160, 290, 300], dtype=torch.int32, device="cuda")

    def both(t):
        z, tok, adv, old, ref, mask, weight = t
        o = runner.policy_loss(ctx, z, tok, adv, old, logp_ref=ref, mask=mask, token_weight=weight, kl_coef=0.1)
        q = runner.preference_loss(ctx, z, tok, start, mask=mask)
        return [o["loss"], o["d_logits"], q["loss"], q["margin"], q["d_logits"]]
    want = [both(a), both(b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for s, t in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append(both(t))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, g in zip(want, got) for x, y in zip(w, g))
    graphs, outs = [], []
    for t in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(both(t))
        graphs.append(graph)
    for x, y in zip(a, b):                       # swap the inputs
        keep = x.clone()
        x.copy_(y)
        y.copy_(keep)
    for s, graph in zip(streams, graphs):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, g in zip(reversed(want), outs) for x, y in zip(w, g))


def test_refusals(ctx):
    z, tok, adv, old, ref, mask, weight = make(4, 64, BF, 1)
    start = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    pol = lambda **k: runner.policy_loss(ctx, **{**dict(logits=z, tokens=tok, advantages=adv, logp_old=old), **k})
    pre = lambda **k: runner.preference_loss(ctx, **{**dict(logits=z, tokens=tok, seq_start=start), **k})
    odd = torch.zeros((4, 65), device="cuda", dtype=BF)
    bad = [
        (lambda: pol(logits=z.half()), "bfloat16 or float32"), (lambda: pol(logits=z[0]), r"\[T, V\]"), (lambda: pol(logits=z.t()), "contiguous rows|tokens"),
        (lambda: pol(logits=z[:1].expand(4, 64)), "overlap"), (lambda: pol(logits=odd), "16 bytes"), (lambda: pol(logits=odd[:, 1:]), "16"),
        (lambda: pol(tokens=tok.long()), "tokens"), (lambda: pol(tokens=tok[:3]), "tokens"), (lambda: pol(mask=mask.bool()), "mask"),
        (lambda: pol(advantages=adv.double()), "advantages"), (lambda: pol(logp_old=None), "'NoneType'|logp_old"), (lambda: pol(logp_ref=ref[:3]), "logp_ref"),
        (lambda: pol(token_weight=weight.half()), "token_weight"), (lambda: pol(n_valid=-1), "n_valid"), (lambda: pol(eps_lo=1.5), "eps_lo"),
        (lambda: pol(eps_hi=-0.1), "eps_hi"), (lambda: pol(eps_hi=float("inf")), "eps_hi"), (lambda: pol(kl_coef=float("nan")), "kl_coef"),
        (lambda: pol(temperature=-1.0), "temperature"), (lambda: pol(temperature=1e-5), "temperature"), (lambda: pol(grad_out=float("inf")), "grad_out"),
        (lambda: pol(d_logits=z.float()), "d_logits"), (lambda: pol(d_logits=z[:3]), "d_logits"), (lambda: pol(logits=z.cpu()), "context is on"),
        (lambda: pre(seq_start=start[:2]), "seq_start"), (lambda: pre(seq_start=start.long()), "seq_start"), (lambda: pre(ref_logp=ref[:3]), "ref_logp"),
        (lambda: pre(beta=float("inf")), "beta"), (lambda: pre(margin=float("nan")), "margin"), (lambda: pre(label_smoothing=1.1), "label_smoothing"),
        (lambda: pre(logits=z[:0], tokens=tok[:0]), "pairs without rows"),
    ]
    for call, text in bad:
        with pytest.raises((B.JackpotError, AttributeError), match=text):
            call()
    # the C entries' own checks
    d = B.jp_policy_desc(T=4, V=64, dtype=B.JP_BF16, eps_lo=0.2, eps_hi=0.2)
    need = B.jp_policy_workspace_bytes(ctx, 4)
    ws, loss = torch.empty(need + 256, dtype=torch.uint8, device="cuda"), torch.empty(3, device="cuda")
    call = lambda desc, w, dz=None, lo=loss: B.jp_policy_loss(ctx, desc, z, tok, mask, adv, old, None, None, lo, None, None, None, dz, w)
    with pytest.raises(B.JackpotError, match="workspace"):
        call(d, ws[:need - 1])
    with pytest.raises(B.JackpotError, match="256-byte"):
        call(d, ws[8:])
    with pytest.raises(B.JackpotError, match="out_loss"):
        call(d, ws, lo=None)
    for field, value in (("T", -1), ("V", 0), ("ld", 63), ("dtype", 2), ("ld_d", 32)):
        e = B.jp_policy_desc(T=4, V=64, dtype=B.JP_BF16)
        setattr(e, field, value)
        with pytest.raises(B.JackpotError):
            call(e, ws, dz=torch.empty_like(z))
    with pytest.raises(B.JackpotError, match="pitch"):
        call(B.jp_policy_desc(T=4, V=64, ld=64, ld_d=72, dtype=B.JP_BF16), ws, dz=z)
    e = B.jp_preference_desc(T=4, V=64, P=2, dtype=B.JP_BF16, flags=2)
    with pytest.raises(B.JackpotError, match="flag"):
        B.jp_preference_loss(ctx, e, z, tok, mask, start, None, loss, None, None, None, None, None, ws)
    call(d, ws)                                                                         # the context works as before
    torch.cuda.synchronize()
