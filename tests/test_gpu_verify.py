"""Verification of drafted tokens (jp_verify_draft) against the sequential procedure in 64 bits.

Accepted counts and tokens must be equal.  Bars of the fp32 outputs: a row's sum of exponentials is taken in fp32 terms whose
exponent (at most 128 in magnitude where it counts, in units of log 2) is rounded twice, 2 * 2^-18 ln 2 = 5.3e-6, with the
exponential's own 2^-22 and 3 * 2^-24 of three sums: below 6e-6 for a log-probability, 1.2e-5 relative for an acceptance
probability (two rows); each is rounded once more to fp32 (by 2^-24 of its value, or by 2^-150, half of fp32's smallest step, next to zero)."""
import math

import numpy as np
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
LOW = {torch.bfloat16: torch.finfo(torch.bfloat16).min, torch.float32: torch.finfo(torch.float32).min}


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def make(n_seq, N, V, dtype, seed, draft=True, sigma=0.7, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = ld or (V + 7) // 8 * 8
    target = torch.full((n_seq, N + 1, ld), 99.0, device="cuda").to(dtype)
    z = torch.randn((n_seq, N + 1, V), generator=g, device="cuda") * 2.5
    target[:, :, :V] = z.to(dtype)
    zd = z[:, :N] + sigma * torch.randn((n_seq, N, V), generator=g, device="cuda")
    dl = torch.full((n_seq, N, ld), 99.0, device="cuda").to(dtype)
    dl[:, :, :V] = zd.to(dtype)
    noise = -torch.log(-torch.log(torch.rand((n_seq, N, V), generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    tok = (zd + noise).argmax(2).to(torch.int32) if N else torch.empty((n_seq, 0), dtype=torch.int32, device="cuda")
    return dict(target_logits=target[:, :, :V], draft_logits=dl[:, :, :V] if draft else None, draft_tokens=tok,
                u_accept=torch.rand((n_seq, N), generator=g, device="cuda"),
                u_sample=torch.rand(n_seq, generator=g, device="cuda"))


def log_softmax(z, t):
    """Of one row in 64 bits; None for a row with NaN or +inf or nothing above -inf."""
    z = z.astype(np.float64) / t
    m = z.max()
    if not np.isfinite(m):
        return None
    with np.errstate(under="ignore"):
        return (z - m) - math.log(np.exp(z - m).sum())       # (differences first: rows of the lowest value)


def first_beyond(mass, u):
    c = np.cumsum(mass)
    return min(int(np.searchsorted(c, u * c[-1], side="right")), int(np.nonzero(mass)[0][-1]))


def one_sequence(zt, zd, tok, u, us, n, t):
    """The procedure, one draft after the other: m, tokens, acceptance probabilities, log-probabilities."""
    N, V = len(tok), zt.shape[1]
    probs, logp, out = np.zeros(N), np.zeros(N + 1), -np.ones(N + 1, np.int64)
    if not (t == 0 or np.float32(1e-4) <= np.float32(t) <= np.float32(1e4)):
        return 0, out, probs, logp
    n = min(max(n, 0), N)
    m, mass = 0, None
    lp = log_softmax(zt[0], t or 1.0)
    while m < n:
        x, lp = tok[m], log_softmax(zt[m], t or 1.0)
        lq = log_softmax(zd[m], t) if zd is not None and t != 0 else None
        draft_bad = zd is not None and t != 0 and lq is None
        a = 0.0
        if lp is not None and not draft_bad and 0 <= x < V:
            if t == 0:
                a = float(x == int(np.argmax(zt[m])))
            elif lp[x] > -840 * math.log(2):                  # (below: probability 0)
                a = math.exp(lp[x]) if lq is None else (np.inf if lq[x] == -np.inf else math.exp(min(lp[x] - lq[x], 700)))
        probs[m] = min(a, 1.0)
        if float(u[m]) < a:
            out[m], logp[m] = x, lp[x]
            m += 1
            continue
        if lp is None or draft_bad:
            return m, out, probs, logp
        p = np.exp(lp)
        if zd is None:
            mass = p.copy()
            if 0 <= x < V:
                mass[x] = 0
        elif t != 0:
            mass = np.maximum(p - np.exp(lq), 0)
        break
    lp = log_softmax(zt[m], t or 1.0)
    if lp is None:
        return m, out, probs, logp
    if t == 0:
        v = int(np.argmax(zt[m]))
    else:
        if mass is None or not mass.sum() > 0:
            mass = np.exp(lp)
        v = first_beyond(mass, float(us) if us > 0 else 0.0)
    out[m], logp[m] = v, lp[v]
    return m, out, probs, logp


def host(t):
    return None if t is None else t.detach().float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def check(ctx, s, n_draft=None, temperature=None):
    out = runner.verify_draft(ctx, **s, n_draft=n_draft, temperature=temperature)
    torch.cuda.synchronize()
    zt, zd, tok, u, us = (host(s[k]) for k in ("target_logits", "draft_logits", "draft_tokens", "u_accept", "u_sample"))
    got = {k: v.cpu().numpy() for k, v in out.items()}
    nd, te = host(n_draft), host(temperature)
    for b in range(zt.shape[0]):
        N = tok.shape[1]
        m, toks, probs, logp = one_sequence(zt[b], None if zd is None else zd[b], tok[b], u[b], us[b],
                                            N if nd is None else int(nd[b]), 1.0 if te is None else float(te[b]))
        assert got["n_accepted"][b] == m, (b, got["n_accepted"][b], m, probs, u[b])
        assert (got["tokens"][b] == toks).all(), (b, got["tokens"][b], toks)
        assert (np.abs(got["accept_prob"][b] - probs) <= (1.2e-5 + U) * probs + 2.0 ** -150).all(), (got["accept_prob"][b], probs)
        with np.errstate(over="ignore", invalid="ignore"):    # (what lies beyond fp32 rounds to its infinity)
            near = np.abs(got["logp"][b] - logp) <= 6e-6 + U * np.abs(logp)
            assert (near | (got["logp"][b] == logp.astype(np.float32))).all(), (got["logp"][b], logp)
    return got


@pytest.mark.parametrize("n_seq,N,V", [(1, 1, 1), (1, 3, 2), (2, 2, 7), (3, 4, 8), (5, 1, 9), (4, 5, 100), (2, 32, 333), (9, 3, 1000),
                                       (1, 4, 4097), (6, 7, 20011), (1, 1, 151936), (3, 4, 151936), (200, 2, 515)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("draft", [True, False])
def test_matches_the_procedure(ctx, n_seq, N, V, dtype, draft):
    check(ctx, make(n_seq, N, V, dtype, seed=n_seq * 31 + N + V, draft=draft))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("draft", [True, False])
def test_ragged_drafts_and_temperatures(ctx, dtype, draft):
    s = make(24, 6, 3001, dtype, seed=5, draft=draft)
    n = torch.arange(24, device="cuda", dtype=torch.int32) % 9 - 1           # -1 .. 7: clamped to 0 .. 6
    t = torch.tensor([1.0, 0.0, 0.3, 2.0, 1e-4, 1e4, 0.01, -1.0, float("nan"), float("inf"), 1e-5, 0.7], device="cuda").repeat(2)
    got = check(ctx, s, n_draft=n, temperature=t)
    assert (got["tokens"][7:11, 0] == -1).all() and (got["n_accepted"][7:11] == 0).all()


def test_without_drafts_it_samples(ctx):
    s = make(40, 0, 5003, torch.float32, seed=3)
    check(ctx, s, temperature=torch.linspace(0, 2, 40, device="cuda"))
    s["draft_logits"] = None
    check(ctx, s)
    s = make(40, 3, 5003, torch.float32, seed=4)
    check(ctx, s, n_draft=torch.zeros(40, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_masked_vocabularies(ctx, dtype):
    """-inf, the type's lowest value, a row with one entry left, rows with nothing left, a row of lowest values only."""
    s = make(12, 3, 2000, dtype, seed=6)
    t, d = s["target_logits"], s["draft_logits"]
    t[0, :, ::3] = d[0, :, ::3] = -math.inf
    t[1, :, :1990] = d[1, :, :1990] = -math.inf
    t[2, :, 100:] = d[2, :, 100:] = LOW[dtype]
    t[3], d[3] = LOW[dtype], LOW[dtype]
    t[4, 0], d[4, 0] = -math.inf, -math.inf
    t[4, 0, 77] = d[4, 0, 77] = -3.0
    s["draft_tokens"][4, 0] = 77
    t[5, 1] = -math.inf                                       # nothing left in a target row
    d[6, 0] = -math.inf                                       # nothing left in a draft row
    t[7, :, :8] = LOW[dtype]                                  # the first entries say nothing of the rest
    t[8, :, 0] = 1000.0
    d[8, :, 0] = 1000.0
    t[9, :, 1999] = 3000.0
    t[10, :, 5:] = -math.inf                                  # the draft's token has probability 0 under the target
    d[11, :, 50] = -math.inf                                  # ... and under the draft
    s["draft_tokens"][11] = 50
    check(ctx, s)
    check(ctx, s, temperature=torch.full((12,), 0.5, device="cuda"))
    check(ctx, s, temperature=torch.zeros(12, device="cuda"))


@pytest.mark.parametrize("offset", [-5000.0, -100.0, 85.0, 5000.0, 1e7])
def test_rows_far_from_zero(ctx, offset):
    s = make(4, 3, 999, torch.float32, seed=7)
    s["target_logits"] += offset
    s["draft_logits"] -= offset
    check(ctx, s)


def test_bad_rows_touch_their_sequence_only(ctx):
    s = make(10, 3, 1500, torch.bfloat16, seed=8)
    clean = check(ctx, s)
    s["target_logits"][2, 0, 40] = math.nan
    s["target_logits"][4, 3, 9] = math.inf
    s["draft_logits"][6, 0, 1499] = math.nan
    s["draft_tokens"][7, 0], s["draft_tokens"][8, 1] = 1500, -7
    got = check(ctx, s)
    assert got["tokens"][2, 0] == -1 and got["n_accepted"][2] == 0
    for b in (0, 1, 3, 5, 9):
        assert all((got[k][b] == clean[k][b]).all() for k in got)
    zero = torch.zeros(10, device="cuda")
    check(ctx, s, temperature=zero)


def test_ends_of_the_random_numbers(ctx):
    s = make(16, 2, 700, torch.float32, seed=9)
    s["target_logits"][8:, :, 0] = -math.inf
    s["target_logits"][8:, :, 699] = -math.inf
    s["u_sample"][0::4], s["u_sample"][1::4] = 0.0, 1 - U
    s["u_accept"][:, 0], s["u_accept"][4:8, 1], s["u_accept"][8:, 1] = 0.0, 1 - U, 0.999
    check(ctx, s)
    s["u_sample"][:] = 1.0                                    # outside the range: the last token with any mass
    got = check(ctx, s)
    assert (got["tokens"] != 0)[8:].all()


def test_greedy_takes_the_lowest_of_equal_entries(ctx):
    s = make(6, 2, 640, torch.bfloat16, seed=10)
    s["target_logits"][:] = s["target_logits"].clamp(max=3.0)  # many entries share the maximum
    z = host(s["target_logits"])
    s["draft_tokens"][:] = torch.tensor(z[:, :2].argmax(2), device="cuda", dtype=torch.int32)
    s["draft_tokens"][3, 1] += 1
    s["target_logits"][5] = -0.0
    s["target_logits"][5, :, 300:] = 0.0                      # -0 and 0 are equal
    s["draft_tokens"][5] = 0
    got = check(ctx, s, temperature=torch.zeros(6, device="cuda"))
    assert list(got["n_accepted"]) == [2, 2, 2, 1, 2, 2]


def test_an_equal_draft_is_always_accepted(ctx):
    s = make(64, 4, 3000, torch.bfloat16, seed=11)
    s["draft_logits"].copy_(s["target_logits"][:, :4])
    s["u_accept"][:] = 1 - U
    got = check(ctx, s)
    assert (got["n_accepted"] == 4).all()


def test_decisions_next_to_their_border(ctx):
    """u_accept on either side of the acceptance probability by one fp32 step: decided as in 64 bits."""
    s = make(60, 1, 4000, torch.bfloat16, seed=12, sigma=1.5)
    zt, zd, tok = host(s["target_logits"]), host(s["draft_logits"]), host(s["draft_tokens"])
    for b in range(60):
        a = math.exp(min(0.0, log_softmax(zt[b, 0], 1)[tok[b, 0]] - log_softmax(zd[b, 0], 1)[tok[b, 0]]))
        u = np.float32(a)
        s["u_accept"][b, 0] = float(np.nextafter(u, np.float32(0 if b % 2 else 1)))
    check(ctx, s)


def test_emitted_tokens_follow_the_target(ctx):
    """60000 sequences of one draft over 6 tokens: the first emitted token has the target's distribution, whatever the draft's."""
    g = torch.Generator(device="cuda").manual_seed(13)
    n, V = 60000, 6
    zt = torch.tensor([0.3, -1.0, 1.2, 0.0, -0.5, 0.8, 0, 0], device="cuda")
    zd = torch.tensor([1.3, 0.5, -0.7, 0.2, 0.5, -0.8, 0, 0], device="cuda")
    tok = torch.multinomial(zd[:V].softmax(0), n, replacement=True, generator=g).to(torch.int32)[:, None]
    out = runner.verify_draft(ctx, zt.expand(n, 2, 8).contiguous()[:, :, :V], zd.expand(n, 1, 8).contiguous()[:, :, :V], tok,
                              torch.rand((n, 1), generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda"))
    freq = torch.bincount(out["tokens"][:, 0].long(), minlength=V).double() / n
    p = zt[:V].double().softmax(0)
    assert ((freq - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n)).all()      # five standard deviations
    # the overlap of the two distributions is accepted
    want = float(torch.minimum(p, zd[:V].double().softmax(0)).sum())
    assert abs(float(out["n_accepted"].double().mean()) - want) <= 5 * math.sqrt(want * (1 - want) / n)


def test_pitches_streams_graphs_and_dirty_scratch(ctx):
    s = make(7, 3, 1001, torch.bfloat16, seed=14, ld=1040)
    first = check(ctx, s)
    wide = torch.full((7, 6, 1040), 50.0, device="cuda", dtype=torch.bfloat16)
    wide[:, 1:5, :1001] = s["target_logits"]                  # sequences further apart than their rows
    s2 = dict(s, target_logits=wide[:, 1:5, :1001])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = runner.verify_draft(ctx, **s2)
    side.synchronize()
    assert all((first[k] == second[k].cpu().numpy()).all() for k in first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = runner.verify_draft(ctx, **s)
    for _ in range(3):
        s["u_sample"].copy_(torch.rand(7, device="cuda"))
        s["u_accept"].copy_(torch.rand((7, 3), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        now = check(ctx, s)
        assert all((now[k] == third[k].cpu().numpy()).all() for k in now)
    # the C entry with scratch full of ones, twice
    d = B.jp_verify_desc(B=7, V=1001, N=3, dtype=B.JP_BF16, ld_target=1040, ld_draft=1040)
    ws = torch.full((B.jp_verify_workspace_bytes(ctx, 7, 3, 1001, B.JP_BF16, True),), 255, dtype=torch.uint8, device="cuda")
    n_acc = torch.empty(7, dtype=torch.int32, device="cuda")
    toks = torch.empty((7, 4), dtype=torch.int32, device="cuda")
    for _ in range(2):
        B.jp_verify_draft(ctx, d, s["target_logits"], s["draft_logits"], s["draft_tokens"], None, None, s["u_accept"],
                          s["u_sample"], n_acc, toks, None, None, ws)
        assert (toks.cpu().numpy() == now["tokens"]).all() and (n_acc.cpu().numpy() == now["n_accepted"]).all()


def test_refusals(ctx):
    s = make(3, 2, 64, torch.bfloat16, seed=1)
    bad = [
        (dict(target_logits=s["target_logits"].half()), "bfloat16 or float32"),
        (dict(draft_logits=s["draft_logits"].float()), "dtype"),
        (dict(draft_logits=s["draft_logits"][:, :1]), "draft_logits"),
        (dict(draft_tokens=s["draft_tokens"].long()), "draft_tokens"),
        (dict(draft_tokens=s["draft_tokens"][:2]), "draft_tokens"),
        (dict(u_accept=s["u_accept"].double()), "u_accept"),
        (dict(u_sample=s["u_sample"][:2]), "u_sample"),
        (dict(n_draft=torch.ones(2, dtype=torch.int32, device="cuda")), "n_draft"),
        (dict(temperature=torch.ones(3, dtype=torch.float64, device="cuda")), "temperature"),
        (dict(target_logits=s["target_logits"][:1].expand(3, 3, 64)), "overlap"),
        (dict(target_logits=s["target_logits"].transpose(1, 2)), "u_accept|draft_logits|contiguous"),
        (dict(target_logits=s["target_logits"].cpu()), "context is on"),
        (dict(u_sample=s["u_sample"].cpu()), "context is on"),
    ]
    for change, text in bad:
        with pytest.raises(B.JackpotError, match=text):
            runner.verify_draft(ctx, **{**s, **change})
    odd = make(2, 1, 63, torch.bfloat16, seed=2, ld=63)
    with pytest.raises(B.JackpotError, match="16 bytes"):
        runner.verify_draft(ctx, **odd)
    with pytest.raises(B.JackpotError, match="MAX_DRAFT"):
        runner.verify_draft(ctx, **make(1, 33, 16, torch.bfloat16, seed=2))
    empty = runner.verify_draft(ctx, **make(0, 2, 64, torch.bfloat16, seed=2))
    assert empty["tokens"].shape == (0, 3)
    d = B.jp_verify_desc(B=3, V=64, N=2, dtype=B.JP_BF16)
    ws = torch.empty(B.jp_verify_workspace_bytes(ctx, 3, 2, 64, B.JP_BF16, True), dtype=torch.uint8, device="cuda")
    n_acc = torch.empty(3, dtype=torch.int32, device="cuda")
    toks = torch.empty((3, 3), dtype=torch.int32, device="cuda")
    tail = (s["draft_tokens"], None, None, s["u_accept"], s["u_sample"], n_acc, toks, None, None)
    t, q = s["target_logits"], s["draft_logits"]
    with pytest.raises(B.JackpotError, match="workspace"):
        B.jp_verify_draft(ctx, d, t, q, *tail, ws[:-1])
    with pytest.raises(B.JackpotError, match="workspace"):
        B.jp_verify_draft(ctx, d, t, q, *tail, None)
    with pytest.raises(B.JackpotError, match="NULL"):
        B.jp_verify_draft(ctx, d, None, q, *tail, ws)
    for field, value in (("B", -1), ("B", 65536), ("V", 0), ("N", 33), ("N", -1), ("dtype", 2), ("ld_target", 56), ("seq_draft", 4)):
        e = B.jp_verify_desc(B=3, V=64, N=2, dtype=B.JP_BF16)
        setattr(e, field, value)
        with pytest.raises(B.JackpotError):
            B.jp_verify_draft(ctx, e, t, q, *tail, ws)
    check(ctx, s)


def draws_inside_entries(s, rng):
    """Sets u_sample to the middle of what an entry of more than average mass takes of the first row's max(p - q, 0), a random one a sequence."""
    zt, zd = host(s["target_logits"]), host(s["draft_logits"])
    for b in range(zt.shape[0]):
        mass = np.maximum(np.exp(log_softmax(zt[b, 0], 1)) - np.exp(log_softmax(zd[b, 0], 1)), 0)
        c = np.cumsum(mass)
        v = rng.choice(np.nonzero(mass >= c[-1] / mass.size)[0])
        s["u_sample"][b] = float((c[v] - mass[v] / 2) / c[-1])


@pytest.mark.parametrize("V", [1000, 20011])
@pytest.mark.parametrize("eps", [1e-5, 1e-6, 1e-7])
def test_draws_between_nearly_equal_rows(ctx, V, eps):
    """A draft that differs from the target by little more than fp32's steps: p - q is far below what the sums of the first pass are
    good to.  The draw is half an entry's mass from its borders, at least 1 / 2 V of the whole: above 2e-5, where p and q in 64 bits, off by
    2e-16 each, leave 2e-16 sqrt(V) / 1e-8 of a whole of 1e-8 and more."""
    s = make(100, 1, V, torch.float32, seed=21)
    g = torch.Generator(device="cuda").manual_seed(22)
    s["draft_logits"].copy_(s["target_logits"][:, :1] + eps * torch.randn((100, 1, V), generator=g, device="cuda"))
    s["draft_tokens"][:] = -1                                 # rejected
    draws_inside_entries(s, np.random.default_rng(23))
    check(ctx, s)


def test_draws_where_one_entry_is_raised_by_a_step(ctx):
    """Equal rows but for the largest entry, one fp32 step higher in the draft: everything else has p above q, by 1e-7 of itself."""
    s = make(64, 1, 3000, torch.float32, seed=24)
    z = s["target_logits"]
    z[:, :, 7] = 7.5
    z[:, :, 2999] = 11.0
    s["draft_logits"].copy_(z[:, :1])
    s["draft_logits"][:, :, 2999] = float(np.nextafter(np.float32(11.0), np.float32(12)))
    s["draft_tokens"][:] = 3000                               # rejected
    draws_inside_entries(s, np.random.default_rng(25))
    got = check(ctx, s)
    assert (got["tokens"][:, 0] != 2999).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_borders_where_the_start_of_a_slice_is_masked(ctx, dtype):
    """All but the last 1000 entries are masked and these lie near -40: the sums have no reference nearby and are off by up to 3e-6; u_accept
    is one fp32 step from the border all the same."""
    n, V = 60, 50000
    s = make(n, 1, V, dtype, seed=27, sigma=1.0)
    for k in ("target_logits", "draft_logits"):
        s[k] -= 40.0
        s[k][:, :, :V - 1000] = -math.inf
    g = torch.Generator(device="cuda").manual_seed(28)
    s["draft_tokens"][:] = torch.randint(V - 1000, V, (n, 1), generator=g, device="cuda", dtype=torch.int32)
    zt, zd, tok = host(s["target_logits"]), host(s["draft_logits"]), host(s["draft_tokens"])
    for b in range(n):
        a = math.exp(min(0.0, log_softmax(zt[b, 0], 1)[tok[b, 0]] - log_softmax(zd[b, 0], 1)[tok[b, 0]]))
        s["u_accept"][b, 0] = float(np.nextafter(np.float32(a), np.float32(0 if b % 2 else 1)))
    check(ctx, s)


def test_draws_between_nearly_equal_rows_far_from_zero(ctx):
    """Logits near 2^21, a quarter apart: equal rows but for one entry of 1e-8, a step higher in the draft.  Everything else has p above q by
    less than 1e-8 of itself."""
    s = make(64, 1, 3000, torch.float32, seed=29)
    z = s["target_logits"]
    z.copy_((z * 4).round() / 4 + 2.0 ** 21)
    z[:, :, 2000] = z.amax(2) - 12
    s["draft_logits"].copy_(z[:, :1])
    s["draft_logits"][:, :, 2000] += 0.25
    s["draft_tokens"][:] = -5                                 # rejected
    draws_inside_entries(s, np.random.default_rng(30))
    check(ctx, s)
