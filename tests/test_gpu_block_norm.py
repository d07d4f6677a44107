"""The norms around a block (jp_block_norm_forward, jp_block_norm_backward) against a plain implementation in 64 bits.

Bars.  u = 2^-24.  A row's sums add at most 16 terms a thread (H / 1024 for the widest rows: up to 24 here) and a tree of 10 levels: below 32 u of the
sum of magnitudes.  mean is within 32 u of the mean magnitude, rstd within 32 u relative (and the square of the mean's share); the handful of
operations on an element adds a few u.  So 96 u times the magnitudes that enter an output (two norms one behind the other, each with
its sums) bounds the arithmetic, and a rounding adds half a step of its type, 2^-8 for bf16.  The norm in front of the next block is
taken of the sum as stored, so y is held against the call's own sum, and the backward's inputs are exact.  Sums over rows add at
most 32 rows a block here, then every 32nd block's line, then a tree: 128 u of the sum of magnitudes."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: U}
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


FORMS = {                                       # post, gate, token gate, bias
    "plain": (False, False, False, False), "post": (True, False, False, False), "all": (True, True, True, True),
    "gates": (False, True, True, True), "post_gate": (True, True, False, False), "token": (False, False, True, False),
    "post_bias": (True, False, False, True), "gate": (False, True, False, False),
}


def make(T, H, dtype, param, form, seed, ld=None, start=0):
    post, gate, token, bias = FORMS[form]
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = ld or H

    def matrix(scale, shift=0.0):
        flat = torch.full((start + T * ld,), float("nan"), device="cuda", dtype=dtype)
        m = flat[start:].view(T, ld)[:, :H]
        m.copy_((torch.randn((T, H), generator=g, device="cuda") * scale + shift).to(dtype))
        return m

    def vec(at, scale):
        return (at + scale * torch.randn(H, generator=g, device="cuda")).to(param)
    s = dict(x=matrix(0.7, 0.2), residual=matrix(2.0, 0.5), dy=matrix(1.0), dsum=matrix(1.0), weight=vec(1, 0.3), bias=vec(0, 0.2) if bias else None,
             post_weight=vec(1, 0.3) if post else None, post_bias=vec(0, 0.2) if bias and post else None, gate=vec(0.5, 0.3) if gate else None,
             token_gate=torch.rand(T, generator=g, device="cuda") + 0.1 if token else None)
    s["scale"] = 0.75
    return s


def d64(t):
    return None if t is None else t.double()


def norm64(x, rms):
    mean = torch.zeros(x.shape[0], dtype=torch.float64, device=x.device) if rms else x.mean(1)
    d = x - mean[:, None]
    return mean, 1 / torch.sqrt((d * d).mean(1) + EPS)


def branch(s, mean, rstd):
    """xhat, u and the factor of each element, from the statistics given."""
    x = s["x"].double()
    xh, u = x, x
    if s["post_weight"] is not None:
        xh = (x - (0 if mean is None else mean.double()[:, None])) * rstd.double()[:, None]
        u = xh * d64(s["post_weight"]) + (0 if s["post_bias"] is None else d64(s["post_bias"]))
    f = torch.full_like(x, s["scale"])
    if s["gate"] is not None:
        f = f * d64(s["gate"])
    if s["token_gate"] is not None:
        f = f * d64(s["token_gate"])[:, None]
    return xh, u, f


def check_forward(o, s, rms, residual, c=96):
    dtype = s["x"].dtype
    x = s["x"].double()
    m1, r1 = norm64(x, rms)
    _, u, f = branch(s, m1, r1)
    want = residual.double() + f * u
    mag = residual.double().abs() + f.abs() * (u.abs() if s["post_weight"] is None else
                                               (x.abs() + x.abs().mean(1, keepdim=True)) * r1[:, None] * d64(s["post_weight"]).abs() + u.abs())
    assert ((o["sum"].double() - want).abs() <= HALF[dtype] * want.abs() * (1 + 2.0 ** -8) + c * U * mag).all()
    if s["post_weight"] is not None:
        assert ((o["post_rstd"].double() - r1).abs() <= c * U * r1 * (1 + (x.abs().mean(1) * r1) ** 2)).all()
        assert rms or ((o["post_mean"].double() - m1).abs() <= c * U * x.abs().mean(1)).all()
    t = o["sum"].double()                        # as stored
    m2, r2 = norm64(t, rms)
    y = (t - m2[:, None]) * r2[:, None] * d64(s["weight"]) + (0 if s["bias"] is None else d64(s["bias"]))
    mag = (t.abs() + t.abs().mean(1, keepdim=True)) * r2[:, None] * d64(s["weight"]).abs() + y.abs()
    assert ((o["y"].double() - y).abs() <= HALF[dtype] * y.abs() * (1 + 2.0 ** -8) + c * U * mag).all()
    assert ((o["rstd"].double() - r2).abs() <= c * U * r2 * (1 + (t.abs().mean(1) * r2) ** 2)).all()
    assert rms or ((o["mean"].double() - m2).abs() <= c * U * t.abs().mean(1)).all()


def norm_bwd64(g, xh, rstd, rms):
    dx = g - xh * (g * xh).mean(1, keepdim=True) - (0 if rms else g.mean(1, keepdim=True))
    mag = g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True) + g.abs().mean(1, keepdim=True)
    return dx * rstd, mag * rstd


def check_backward(o, s, f, total, rms, dsum, c=96, cs=128):
    dtype = s["x"].dtype
    rstd = d64(f["rstd"])[:, None]
    xh2 = (total.double() - (0 if rms else d64(f["mean"])[:, None])) * rstd
    dy = s["dy"].double()
    ds, mag = norm_bwd64(dy * d64(s["weight"]), xh2, rstd, rms)
    if dsum is not None:
        ds, mag = ds + dsum.double(), mag + dsum.double().abs()

    def near(got, want, mag, k=c):
        half = HALF[dtype] if got.dtype is dtype and got.dim() == 2 else U
        assert ((got.double() - want).abs() <= half * want.abs() * (1 + 2.0 ** -8) + k * U * mag).all()
    near(o["dresidual"], ds, mag)
    near(o["dweight"], (dy * xh2).sum(0), (dy * xh2).abs().sum(0), cs)
    if o["dbias"] is not None:
        near(o["dbias"], dy.sum(0), dy.abs().sum(0), cs)
    xh, u, fac = branch(s, f["post_mean"], f["post_rstd"])
    umag = u.abs() if s["post_weight"] is None else (xh * d64(s["post_weight"])).abs() + (0 if s["post_bias"] is None else d64(s["post_bias"]).abs())
    one = torch.full_like(xh, s["scale"])
    gt = one if s["token_gate"] is None else one * d64(s["token_gate"])[:, None]
    gc = one if s["gate"] is None else one * d64(s["gate"])
    if s["gate"] is not None:
        near(o["dgate"], (gt * u * ds).sum(0), (gt * umag * mag).abs().sum(0), cs + c)
    if s["token_gate"] is not None:
        near(o["dtoken_gate"], (gc * u * ds).sum(1), (gc * umag * mag).abs().sum(1), 2 * c)
    du, dmag = fac * ds, fac.abs() * mag
    if s["post_weight"] is not None:
        near(o["dpost_weight"], (du * xh).sum(0), (dmag * xh.abs()).sum(0), cs + c)
        if o["dpost_bias"] is not None:
            near(o["dpost_bias"], du.sum(0), dmag.sum(0), cs + c)
        w, r = d64(s["post_weight"]), d64(f["post_rstd"])[:, None]
        du, _ = norm_bwd64(du * w, xh, r, rms)
        g = dmag * w.abs()
        dmag = (g + xh.abs() * (g * xh.abs()).mean(1, keepdim=True) + g.mean(1, keepdim=True)) * r
    near(o["dx"], du, dmag, 2 * c)


def arguments(s):
    return {k: s[k] for k in ("post_weight", "post_bias", "gate", "token_gate", "scale")}


def run_forward(ctx, s, rms, **k):
    return runner.block_norm(ctx, s["x"], s["residual"], s["weight"], s["bias"], eps=EPS, rms=rms, **arguments(s), **k)


def run_backward(ctx, s, f, total, rms, dsum, **k):
    return runner.block_norm_backward(ctx, s["dy"], dsum, s["x"], total, s["weight"], f["mean"], f["rstd"], post_mean=f["post_mean"],
                                      post_rstd=f["post_rstd"], rms=rms, **arguments(s), **k)


SHAPES = [(1, 1), (1, 2048), (3, 8), (5, 7), (9, 100), (17, 63), (33, 256), (64, 1283), (7, 2049), (130, 4096), (2, 5120), (6, 8192), (3, 8200),
          (2, 16384), (1000, 512), (5003, 96), (2, 20011), (5, 6152), (9, 4104), (40, 12288)]


@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form,rms", [("all", False), ("post_gate", True), ("plain", True), ("gates", False)])
def test_both_passes_match_the_formula(ctx, T, H, dtype, form, rms):
    s = make(T, H, dtype, F32 if form == "all" else dtype, form, T * 7 + H)
    keep = {k: v.clone() for k, v in s.items() if isinstance(v, torch.Tensor)}
    f = run_forward(ctx, s, rms)
    assert (f["mean"] is None) == rms and (f["post_rstd"] is None) == (s["post_weight"] is None)
    check_forward(f, s, rms, s["residual"])
    dsum = None if form == "plain" else s["dsum"]
    o = run_backward(ctx, s, f, f["sum"], rms, dsum, bias=s["bias"] is not None)
    check_backward(o, s, f, f["sum"], rms, dsum)
    assert all(torch.equal(s[k], v) for k, v in keep.items())
    again = run_backward(ctx, s, f, f["sum"], rms, dsum, bias=s["bias"] is not None)
    assert all(a is b or torch.equal(a, b) for a, b in zip(o.values(), again.values()))


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("T,H,ld,start", [(50, 768, 768, 0), (41, 515, 515, 0), (37, 1000, 1008, 8), (29, 250, 253, 1), (19, 6000, 6001, 3)])
def test_forms_pitches_and_starts(ctx, form, rms, bias, T, H, ld, start):
    for dtype in (BF, F32):
        s = make(T, H, dtype, dtype, form, T + H, ld, start)
        f = run_forward(ctx, s, rms)
        check_forward(f, s, rms, s["residual"])
        o = run_backward(ctx, s, f, f["sum"], rms, s["dsum"], bias=bias)
        assert (o["dbias"] is None) != bias and (o["dpost_bias"] is None) == (s["post_weight"] is None or not bias)
        check_backward(o, s, f, f["sum"], rms, s["dsum"])


@pytest.mark.parametrize("T,H", [(4000, 2048), (3001, 4096), (9001, 40), (2500, 1283), (2100, 8192), (20011, 63), (1999, 5112)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form,rms", [("all", False), ("post", True), ("post_gate", True)])
def test_many_rows(ctx, T, H, dtype, form, rms):
    s = make(T, H, dtype, F32, form, T + H)
    f = run_forward(ctx, s, rms)
    check_forward(f, s, rms, s["residual"])
    o = run_backward(ctx, s, f, f["sum"], rms, s["dsum"], bias=s["bias"] is not None)
    check_backward(o, s, f, f["sum"], rms, s["dsum"], cs=160)


@pytest.mark.parametrize("T,H,ld", [(37, 2048, 2056), (21, 1000, 1001), (9, 63, 70), (5, 20011, 20011), (300, 4096, 4096)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_in_place(ctx, T, H, ld, dtype):
    """Outputs in the inputs' places give what outputs beside them give; nothing beside the rows is written."""
    s = make(T, H, dtype, dtype, "all", 3, ld)
    beside = lambda: torch.empty_strided(s["x"].shape, s["x"].stride(), dtype=dtype, device="cuda")
    f = run_forward(ctx, s, False, out_sum=beside(), out=beside())
    total = f["sum"].clone(memory_format=torch.preserve_format)
    sums = beside()
    sums.copy_(total)
    o = run_backward(ctx, s, f, sums, False, s["dsum"], dx=beside(), dresidual=beside())
    for pair in (("dy", "dsum"), ("x", "sum"), ("sum", "dy")):
        t = {**s, "dy": beside().copy_(s["dy"]), "dsum": beside().copy_(s["dsum"]), "x": beside().copy_(s["x"])}
        t["sum"] = beside().copy_(total)
        q = run_backward(ctx, t, f, t["sum"], False, t["dsum"], dx=t[pair[0]], dresidual=t[pair[1]])
        assert all(torch.equal(o[k], q[k]) for k in o), pair
    x, r = beside().copy_(s["x"]), beside().copy_(s["residual"])
    flat_x = torch.as_strided(x, (T - 1, ld - H), (ld, 1), H) if ld > H else None
    if flat_x is not None:
        flat_x.fill_(7.0)
    g = run_forward(ctx, {**s, "x": x, "residual": r}, False, out_sum=r, out=x)
    assert g["sum"].data_ptr() == r.data_ptr() and torch.equal(r, total) and torch.equal(x, f["y"])
    assert flat_x is None or (flat_x == 7).all()
    x = beside().copy_(s["x"])
    g = run_forward(ctx, {**s, "x": x}, False, out_sum=x, out=beside())
    assert torch.equal(x, total) and torch.equal(g["y"], f["y"])


def test_no_rows(ctx):
    s = make(1, 640, F32, F32, "all", 1)
    s.update({k: s[k][:0] for k in ("x", "residual", "dy", "dsum", "token_gate")})
    f = run_forward(ctx, s, False)
    assert f["sum"].shape == (0, 640) and f["y"].shape == (0, 640)
    o = run_backward(ctx, s, f, f["sum"], False, s["dsum"])
    assert o["dx"].shape == (0, 640) and all((o[k] == 0).all() for k in ("dweight", "dbias", "dpost_weight", "dpost_bias", "dgate"))


def test_rows_do_not_touch_one_another(ctx):
    s = make(12, 768, F32, F32, "all", 4)
    s["x"][3], s["residual"][5], s["x"][8] = float("nan"), float("inf"), 0.0
    f = run_forward(ctx, s, False)
    good = [i for i in range(12) if i not in (3, 5)]
    sub = {k: (v[good] if isinstance(v, torch.Tensor) and v.shape[0] == 12 else v) for k, v in s.items()}
    check_forward({k: v[good] for k, v in f.items()}, sub, False, sub["residual"])
    o = run_backward(ctx, s, f, f["sum"], False, s["dsum"])
    assert o["dx"][good].isfinite().all() and o["dresidual"][good].isfinite().all()


@pytest.mark.parametrize("T,H", [(23, 7), (40, 63), (21, 515), (600, 1283), (1301, 2047), (30, 4097)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form,rms", [("all", False), ("post_gate", True)])
def test_packed_odd_rows_do_not_touch_one_another(ctx, T, H, dtype, form, rms):
    """Rows that share 16 bytes with a row of NaN give the bits that they give beside a row of zeros."""
    s = make(T, H, dtype, dtype, form, T + H)
    bad, good = slice(1, None, 2), slice(0, None, 2)
    clean, f = [], None
    for value in (0.0, float("nan")):
        t = {**s, "x": s["x"].clone(), "residual": s["residual"].clone()}
        t["x"][bad], t["residual"][bad] = value, value
        o = run_forward(ctx, t, rms)
        f = f or o
        clean.append([o[k][good] for k in ("sum", "y", "rstd", "post_rstd")])
    assert all(torch.equal(a, b) for a, b in zip(*clean))
    grads = []
    for value in (0.0, float("nan")):
        t = {**s, **{k: s[k].clone() for k in ("dy", "dsum", "x")}, "sum": f["sum"].clone()}
        for k in ("dy", "dsum", "x", "sum"):
            t[k][bad] = value
        o = run_backward(ctx, t, f, t["sum"], rms, t["dsum"], bias=s["bias"] is not None)
        grads.append([o[k][good] for k in ("dx", "dresidual")] + ([] if o["dtoken_gate"] is None else [o["dtoken_gate"][good]]))
    assert all(torch.equal(a, b) for a, b in zip(*grads)) and grads[0][0].isfinite().all()


@pytest.mark.parametrize("T,H", [(2500, 2047), (1300, 2500), (1300, 2560), (1300, 4097), (700, 4600), (650, 5112)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form,rms", [("all", False), ("plain", True), ("post_gate", True)])
def test_widths_of_larger_blocks(ctx, T, H, dtype, form, rms):
    s = make(T, H, dtype, dtype, form, T + H)
    f = run_forward(ctx, s, rms)
    check_forward(f, s, rms, s["residual"])
    dsum = None if form == "plain" else s["dsum"]
    o = run_backward(ctx, s, f, f["sum"], rms, dsum, bias=s["bias"] is not None)
    check_backward(o, s, f, f["sum"], rms, dsum, cs=160)


def test_gradients_against_differences(ctx):
    T, H, h = 3, 21, 1e-5
    for rms in (False, True):
        s = make(T, H, F32, F32, "all", 9)
        f = run_forward(ctx, s, rms)
        total = f["sum"]
        o = run_backward(ctx, s, f, total, rms, s["dsum"])

        def loss(t):
            """dsum and dy are the gradients that arrive at sum and y, and what comes after them is linear."""
            t = {k: d64(v) if isinstance(v, torch.Tensor) else v for k, v in t.items()}
            m1, r1 = norm64(t["x"], rms)
            _, u, fac = branch(t, m1, r1)
            total = t["residual"] + fac * u
            m2, r2 = norm64(total, rms)
            y = (total - m2[:, None]) * r2[:, None] * t["weight"] + t["bias"]
            return float((t["dsum"] * total + t["dy"] * y).sum())
        for name, grad in (("x", "dx"), ("residual", "dresidual"), ("weight", "dweight"), ("bias", "dbias"), ("post_weight", "dpost_weight"),
                           ("post_bias", "dpost_bias"), ("gate", "dgate"), ("token_gate", "dtoken_gate")):
            flat = s[name].double().reshape(-1)
            for i in range(0, flat.numel(), 4):
                up, down = flat.clone(), flat.clone()
                up[i] += h
                down[i] -= h
                num = (loss({**s, name: up.view(s[name].shape)}) - loss({**s, name: down.view(s[name].shape)})) / (2 * h)
                # differences: h^2 times third derivatives of order 100, and 2^-52 |loss| / h: below 1e-7; the stored sum is
                # half a step, 2^-24 of 5, away from the one of the differences
                assert abs(num - float(o[grad].reshape(-1)[i])) <= 2e-5 * (1 + abs(num)), (name, i)


def test_streams_and_graphs(ctx):
    a, b = make(300, 2048, BF, F32, "all", 1), make(300, 2048, BF, F32, "all", 2)

    def both(s):
        f = run_forward(ctx, s, False)
        o = run_backward(ctx, s, f, f["sum"], False, s["dsum"])
        return [f["sum"], f["y"]] + [v for v in o.values()]
    want = [both(a), both(b)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for st, s in zip(streams, (a, b)):
        with torch.cuda.stream(st):
            got.append(both(s))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, g in zip(want, got) for x, y in zip(w, g))
    graphs, outs = [], []
    for s in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(both(s))
        graphs.append(graph)
    for k in a:                                  # swap the inputs
        if isinstance(a[k], torch.Tensor):
            keep = a[k].clone()
            a[k].copy_(b[k])
            b[k].copy_(keep)
    for st, graph in zip(streams, graphs):
        with torch.cuda.stream(st):
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for w, g in zip(reversed(want), outs) for x, y in zip(w, g))


def test_offsets_beyond_32_bits(ctx):
    """300,000 rows 8000 elements apart: the last rows lie beyond 2^31 elements."""
    T, H, ld = 300000, 64, 8000
    flat = torch.zeros(T * ld, device="cuda", dtype=BF)
    x = flat.view(T, ld)[:, :H]
    r = flat.view(T, ld)[:, 512:512 + H]
    g = torch.Generator(device="cuda").manual_seed(3)
    x.copy_(torch.randn((T, H), generator=g, device="cuda").to(BF))
    r.copy_(torch.randn((T, H), generator=g, device="cuda").to(BF))
    w = torch.rand(H, generator=g, device="cuda") + 0.5
    f = runner.block_norm(ctx, x, r, w, post_weight=w, rms=True, eps=EPS)
    s = dict(x=x[-50:], residual=r[-50:], weight=w, bias=None, post_weight=w, post_bias=None, gate=None, token_gate=None, scale=1.0)
    check_forward({k: (None if v is None else v[-50:]) for k, v in f.items()}, s, True, r[-50:])
    o = runner.block_norm_backward(ctx, x, None, x, r, w, None, f["rstd"], post_weight=w, post_rstd=f["post_rstd"], rms=True, bias=False)
    p = runner.block_norm_backward(ctx, x[-50:].contiguous(), None, x[-50:].contiguous(), r[-50:].contiguous(), w, None, f["rstd"][-50:].contiguous(),
                                   post_weight=w, post_rstd=f["post_rstd"][-50:].contiguous(), rms=True, bias=False)
    assert torch.equal(o["dx"][-50:], p["dx"]) and torch.equal(o["dresidual"][-50:], p["dresidual"])


def test_refusals(ctx):
    s = make(4, 64, BF, BF, "all", 1)
    f = run_forward(ctx, s, False)
    fwd = lambda **k: run_forward(ctx, {**s, **{n: v for n, v in k.items() if n in s}}, False, **{n: v for n, v in k.items() if n not in s})
    def bwd(**k):
        t, u = {**s, **{n: v for n, v in k.items() if n in s}}, {**f, **{n: v for n, v in k.items() if n in f and n not in s}}
        return run_backward(ctx, t, u, u["sum"], False, t["dsum"], **{n: v for n, v in k.items() if n not in s and n not in f})
    bad = [
        (lambda: fwd(x=s["x"].half()), "bfloat16 or float32|dtype"), (lambda: fwd(residual=s["residual"].float()), "residual"),
        (lambda: fwd(residual=s["residual"][:3]), "residual"), (lambda: fwd(weight=s["weight"][:63]), "weight"), (lambda: fwd(bias=s["bias"].float()), "bias"),
        (lambda: fwd(post_weight=s["post_weight"].float()), "post_weight"), (lambda: fwd(gate=s["gate"][1:]), "gate"),
        (lambda: fwd(token_gate=s["token_gate"].double()), "token_gate"), (lambda: fwd(post_weight=None), "post_bias"), (lambda: fwd(scale=float("inf")), "scale"),
        (lambda: fwd(out=s["x"][:3]), "out"), (lambda: fwd(out_sum=s["x"], out=s["x"]), "same matrix"), (lambda: fwd(x=s["x"].t()), "contiguous rows|shape"),
        (lambda: fwd(residual=s["residual"][:1].expand(4, 64)), "overlap"), (lambda: fwd(residual=s["residual"].cpu()), "context is on"),
        (lambda: bwd(dy=s["dy"].float()), "dy"), (lambda: bwd(sum=f["sum"][:2]), "sum"), (lambda: bwd(rstd=f["rstd"].double()), "rstd"),
        (lambda: bwd(mean=None), "mean"), (lambda: bwd(post_rstd=f["post_rstd"][:2]), "post_rstd"), (lambda: bwd(post_mean=None), "post_mean"),
        (lambda: bwd(dx=s["dy"], dresidual=s["dy"]), "same matrix"), (lambda: bwd(dx=s["x"][:2]), "dx"),
    ]
    for call, text in bad:
        with pytest.raises(B.JackpotError, match=text):
            call()
    # the C entries' own checks
    def desc(**k):
        d = B.jp_block_norm_desc(T=4, H=64, dtype=B.JP_BF16, param_dtype=B.JP_BF16, scale=1.0)
        for n, v in k.items():
            setattr(d, n, v)
        return d
    y, t = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    call = lambda d, **k: B.jp_block_norm_forward(ctx, d, k.get("x", s["x"]), s["residual"], k.get("weight", s["weight"]), None, None, k.get("post_bias"), None, None, t, y,
                                                  None, None, None, None)
    for d, k, text in ((desc(T=-1), {}, "T or H"), (desc(H=0), {}, "T or H"), (desc(ld_x=63), {}, "leading"), (desc(dtype=2), {}, "dtype"), (desc(flags=2), {}, "flag"),
                       (desc(eps=-1.0), {}, "eps"), (desc(scale=float("nan")), {}, "scale"), (desc(), {"weight": None}, "NULL"), (desc(), {"x": None}, "NULL"),
                       (desc(), {"post_bias": s["bias"]}, "post_bias")):
        with pytest.raises(B.JackpotError, match=text):
            call(d, **k)
    need = B.jp_block_norm_workspace_bytes(ctx, 4, 64, B.JP_BF16)
    ws, dw = torch.empty(need + 256, dtype=torch.uint8, device="cuda"), torch.empty(64, device="cuda")
    back = lambda w, x=s["x"], pw=None, dpw=None: B.jp_block_norm_backward(ctx, desc(flags=1), s["dy"], None, x, f["sum"], s["weight"], pw, None, None, None, None, f["rstd"],
                                                                          None, f["rstd"], y, t, dw, None, dpw, None, None, None, w)
    for a, text in (((ws[:need - 1],), "workspace"), ((ws[8:],), "256-byte"), ((ws, None, s["weight"], dw), "x is NULL"), ((ws, s["x"], s["weight"], None), "dpost_weight")):
        with pytest.raises(B.JackpotError, match=text):
            back(*a)
    back(ws, None)                                                                      # without norm and gates x is not needed
    call(desc())                                                                        # the context works as before
    torch.cuda.synchronize()
