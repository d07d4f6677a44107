"""Layer norm and RMS norm (jp_layer_norm_forward, jp_layer_norm_backward) against a plain implementation in 64 bits.

Bars.  u = 2^-24.  A sum over a row adds at most 160 squares in a lane (20 vectors; the sums of x themselves are a tree
of 3 levels, then 20 terms), then a tree of at most 10 levels.  An addition errs by u of the sum so far, which grows from
0 to the whole for terms of one distribution, so 160 of them make 80 u and rstd, which takes half of it, 40 u; mean is
within 32 u of the sum of magnitudes.  The handful of operations on each element adds a few u more.  64 u times the
magnitudes that enter an output (not the output itself, which may cancel) bounds the fp32 arithmetic; the rounding of
the output adds half a step of its type, 2^-8 relative for bf16.  rstd of the backward is an input there.  The sums over
rows add ceil(T / groups) rows in a register, then 8 groups of a block, then every 32nd line, then a tree of 5 levels:
below 100 terms in a row for the sizes here, so 128 u times the sum of magnitudes.  Rows wider than what registers hold add H / 1024 terms a thread instead of 16."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
EPS = 1e-6


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def make(T, H, dtype, param, bias, seed, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = ld or H
    x = torch.full((T, ld), 7.0, device="cuda").to(dtype)
    x[:, :H] = (torch.randn((T, H), generator=g, device="cuda") * 2 + 0.7).to(dtype)
    dy = torch.full((T, ld), 7.0, device="cuda").to(dtype)
    dy[:, :H] = torch.randn((T, H), generator=g, device="cuda").to(dtype)
    w = (1 + 0.3 * torch.randn(H, generator=g, device="cuda")).to(param)
    b = (0.2 * torch.randn(H, generator=g, device="cuda")).to(param) if bias else None
    return x[:, :H], dy[:, :H], w, b


def plain_forward(x, w, b, rms):
    x, w = x.double(), w.double()
    mean = torch.zeros(x.shape[0], dtype=torch.float64, device=x.device) if rms else x.mean(1)
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).mean(1) + EPS)
    y = d * rstd[:, None] * w
    return (y if b is None else y + b.double()), mean, rstd


def plain_backward(dy, x, w, mean, rstd, rms):
    x, dy, w, rstd = x.double(), dy.double(), w.double(), rstd.double()[:, None]
    xh = x * rstd if rms else (x - mean.double()[:, None]) * rstd
    g = dy * w
    dx = g - xh * (g * xh).mean(1, keepdim=True) - (0 if rms else g.mean(1, keepdim=True))
    mag = (g.abs() + xh.abs() * (g * xh).abs().mean(1, keepdim=True) + g.abs().mean(1, keepdim=True)) * rstd
    return dx * rstd, (dy * xh).sum(0), dy.sum(0), mag, (dy * xh).abs().sum(0), dy.abs().sum(0)


def check_forward(y, mean, rstd, x, w, b, rms, c=64):
    ry, rm, rr = plain_forward(x, w, b, rms)
    xd = x.double()
    spread = (xd.abs() + xd.abs().mean(1, keepdim=True)) * rr[:, None] * w.double().abs()
    mag = spread + ry.abs() + (0 if b is None else b.double().abs())
    assert ((y.double() - ry).abs() <= HALF[x.dtype] * ry.abs() + c * U * mag).all()
    if not rms:
        assert ((mean.double() - rm).abs() <= c * U * xd.abs().mean(1)).all()
    assert ((rstd.double() - rr).abs() <= c * U * rr * (1 + (xd.abs().mean(1) * rr) ** 2)).all()


def check_backward(got, dy, x, w, mean, rstd, rms, c=64, cs=128):
    dx, dw, db = got
    rdx, rdw, rdb, mag, magw, magb = plain_backward(dy, x, w, mean, rstd, rms)
    assert ((dx.double() - rdx).abs() <= HALF[x.dtype] * rdx.abs() + c * U * mag).all()
    # (x - mean) of the formula loses nothing of x itself: its magnitudes are |x| and |mean|
    loss = 0 if rms else (dy.double().abs() * (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None]).sum(0)
    assert ((dw.double() - rdw).abs() <= cs * U * magw + 4 * U * loss).all()
    if db is not None:
        assert ((db.double() - rdb).abs() <= cs * U * magb).all()


SHAPES = [(1, 1), (1, 2048), (3, 8), (5, 7), (9, 100), (17, 63), (33, 256), (64, 1283), (7, 2049), (130, 4096), (2, 5120),
          (6, 8192), (3, 8200), (2, 16384), (1000, 512), (5003, 96), (2, 20011)]


@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms,bias", [(False, True), (True, False), (False, False), (True, True)])
def test_both_passes_match_the_formula(ctx, T, H, dtype, rms, bias):
    x, dy, w, b = make(T, H, dtype, torch.float32 if bias else dtype, bias, seed=T * 7 + H)
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms)
    assert (mean is None) == rms
    check_forward(y, mean, rstd, x, w, b, rms)
    got = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms, bias=bias)
    assert (got[2] is None) == (not bias)
    check_backward(got, dy, x, w, mean, rstd, rms)


@pytest.mark.parametrize("T,H", [(1776, 520), (2001, 1024), (1999, 1288), (1777, 2048), (3600, 4096), (1800, 4088), (1790, 8192), (1900, 6152),
                                 (30011, 63), (2500, 4095)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms,bias,param", [(False, True, torch.float32), (True, False, torch.bfloat16)])
def test_many_rows(ctx, T, H, dtype, rms, bias, param):
    """Rows enough to fill every SM several times over.  A register adds at most 26 rows, a sum of lines at most
    19 (592 blocks, every 32nd)."""
    x, dy, w, b = make(T, H, dtype, param, bias, seed=T + H, ld=H + (H % 16))
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms)
    check_forward(y, mean, rstd, x, w, b, rms)
    got = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms, bias=bias)
    check_backward(got, dy, x, w, mean, rstd, rms)
    again = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms, bias=bias)
    assert all(a is c or torch.equal(a, c) for a, c in zip(got, again))
    # in place as out of place, with rows at the same pitch (which decides the order of a row's sums)
    beside, _, _ = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms, out=torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda"))
    check_forward(beside, mean, rstd, x, w, b, rms)
    y2, _, _ = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms, out=x)
    assert torch.equal(y2, beside)


@pytest.mark.parametrize("T,H", [(3, 5), (1, 1023), (40, 255), (5000, 7), (30011, 63), (1790, 519), (2001, 1283), (1999, 2047), (3600, 4095),
                                 (1801, 5113), (1777, 2558), (600, 4089), (400, 8185), (300, 8191), (9, 16377), (1900, 1028)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rms,param,start", [(False, torch.float32, 0), (True, torch.bfloat16, 0), (False, torch.bfloat16, 3)])
def test_rows_that_share_vectors(ctx, T, H, dtype, rms, param, start):
    """Packed rows of odd width, all matrices at the same offset: NaN around the inputs, and what is around the outputs stays."""
    x0, dy0, w, b = make(T, H, dtype, param, not rms, seed=T + H)

    def placed(src):
        flat = torch.full((start + T * H + 9,), float("nan"), device="cuda", dtype=dtype)
        view = flat[start:start + T * H].view(T, H)
        if src is not None:
            view.copy_(src)
        return flat, view

    (_, x), (_, dy), (fy, y), (fdx, dx) = placed(x0), placed(dy0), placed(None), placed(None)
    _, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms, out=y)
    check_forward(y, mean, rstd, x0, w, b, rms)
    got = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms, bias=not rms, dx=dx)
    check_backward(got, dy0, x0, w, mean, rstd, rms)
    for flat in (fy, fdx):
        assert flat[:start].isnan().all() and flat[start + T * H:].isnan().all()
    same = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms, bias=not rms, dx=dy)
    assert all(a is c or torch.equal(a, c) for a, c in zip(got, same))
    same, _, _ = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms, out=x)
    assert torch.equal(same, y)


@pytest.mark.parametrize("H,ld", [(2048, 2056), (1000, 1001), (63, 70), (4096, 4104)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_row_pitches_and_in_place(ctx, H, ld, dtype):
    T = 37
    x, dy, w, b = make(T, H, dtype, dtype, True, seed=3, ld=ld)
    keep_x, keep_dy = x.clone(), dy.clone()
    big = torch.full((T + 2, ld), 5.0, device="cuda", dtype=dtype)
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS, out=big[1:T + 1, :H])
    check_forward(y, mean, rstd, keep_x, w, b, False)
    assert (big[0] == 5).all() and (big[-1] == 5).all() and (big[:, H:] == 5).all()    # nothing beside the rows is written
    # (bits are compared between rows of the same pitch and offset, which decide the order of a row's sums)
    beside = torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda")
    check_backward(runner.layer_norm_backward(ctx, dy, x, w, mean, rstd), keep_dy, x, w, mean, rstd, False)
    got = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=torch.empty_strided(x.shape, x.stride(), dtype=dtype, device="cuda"))
    same = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, dx=dy)                # dx in dy's place
    assert all(torch.equal(a, c) for a, c in zip(got, same)) and same[0].data_ptr() == dy.data_ptr()
    check_backward(same, keep_dy, x, w, mean, rstd, False)
    y3, _, _ = runner.layer_norm(ctx, x, w, b, eps=EPS, out=beside)
    check_forward(y3, mean, rstd, keep_x, w, b, False)
    y2, _, _ = runner.layer_norm(ctx, x, w, b, eps=EPS, out=x)                         # y in x's place
    assert torch.equal(y2, y3) and y2.data_ptr() == x.data_ptr()
    assert (x.storage_offset() == 0) and (torch.as_strided(x, (T, ld - H), (ld, 1), H) == 7).all()


def test_pointers_off_a_16_byte_boundary(ctx):
    T, H = 21, 1024
    x, dy, w, b = make(T, H, torch.bfloat16, torch.bfloat16, True, seed=9)
    flat = torch.empty(T * H + 3, dtype=torch.bfloat16, device="cuda")
    wf = torch.empty(H + 1, dtype=torch.bfloat16, device="cuda")
    xo = flat[3:].view(T, H)
    xo.copy_(x)
    wo = wf[1:]
    wo.copy_(w)
    y, mean, rstd = runner.layer_norm(ctx, xo, wo, b, eps=EPS)
    check_forward(y, mean, rstd, x, w, b, False)
    check_backward(runner.layer_norm_backward(ctx, dy, xo, wo, mean, rstd), dy, x, w, mean, rstd, False)


def test_no_rows(ctx):
    x = torch.empty((0, 640), device="cuda")
    w = torch.ones(640, device="cuda")
    y, mean, rstd = runner.layer_norm(ctx, x, w)
    assert y.shape == (0, 640) and mean.numel() == 0
    dx, dw, db = runner.layer_norm_backward(ctx, x, x, w, mean, rstd)
    assert dx.shape == (0, 640) and (dw == 0).all() and (db == 0).all()


def test_rows_do_not_touch_one_another(ctx):
    """A row of NaN, one of infinities and one of zeros leave the other rows as they are."""
    x, dy, w, b = make(12, 768, torch.float32, torch.float32, True, seed=4)
    x = x.clone()
    x[3], x[5], x[8] = float("nan"), float("inf"), 0.0
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS)
    good = [i for i in range(12) if i not in (3, 5)]
    check_forward(y[good], mean[good], rstd[good], x[good], w, b, False)
    assert torch.equal(y[8], b) and y[3].isnan().all() and y[5].isnan().all()
    dx, _, _ = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd)
    assert dx[good].isfinite().all()


def test_large_values_do_not_cancel(ctx):
    """A common offset of 1000 standard deviations: the squares are taken of x - mean."""
    x, _, w, b = make(40, 2048, torch.float32, torch.float32, True, seed=6)
    x = (x + 2000).contiguous()
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS)
    ry, rm, rr = plain_forward(x, w, b, False)
    # mean is off by at most 32 u 2000 (the sum's bar above); rstd changes with its square only
    off = 32 * U * 2002
    assert ((mean.double() - rm).abs() <= off).all()
    assert ((rstd.double() / rr - 1).abs() <= 64 * U + (off * rr) ** 2).all()
    assert ((y.double() - ry).abs() <= off * rr[:, None] * w.double().abs() * 1.01 + 64 * U * (ry.abs() + b.double().abs() + 2)).all()


def test_gradient_against_differences(ctx):
    T, H = 4, 37
    x, dy, w, b = make(T, H, torch.float32, torch.float32, True, seed=8)
    for rms in (False, True):
        _, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS, rms=rms)
        dx, dw, db = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms)
        loss = lambda xx, ww, bb: (plain_forward(xx, ww, bb, rms)[0] * dy.double()).sum()
        h = 1e-5
        for t, grad in ((x, dx), (w, dw), (b, db)):
            flat = t.double().reshape(-1)
            for i in range(0, flat.numel(), 5):
                up, down = flat.clone(), flat.clone()
                up[i] += h
                down[i] -= h
                args = [[v if s is t else s.double() for s in (x, w, b)] for v in (up.view(t.shape), down.view(t.shape))]
                num = (loss(*args[0]) - loss(*args[1])) / (2 * h)
                # differences: h^2 times third derivatives of order 10, and 2^-52 |loss| / h; both below 1e-7
                assert abs(float(num) - float(grad.reshape(-1)[i])) <= 1e-5 * (1 + abs(float(num)))


def test_same_bits_every_time_on_any_stream_and_in_a_graph(ctx):
    x, dy, w, b = make(777, 2048, torch.bfloat16, torch.float32, True, seed=11)
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS)
    first = (y, mean, rstd) + runner.layer_norm_backward(ctx, dy, x, w, mean, rstd)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y2, m2, r2 = runner.layer_norm(ctx, x, w, b, eps=EPS)
        second = (y2, m2, r2) + runner.layer_norm_backward(ctx, dy, x, w, m2, r2)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, m3, r3 = runner.layer_norm(ctx, x, w, b, eps=EPS)
        third = (y3, m3, r3) + runner.layer_norm_backward(ctx, dy, x, w, m3, r3)
    x.copy_(x.flip(0))
    dy.copy_(dy.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(third[0], first[0].flip(0)) and torch.equal(third[3], first[3].flip(0))


def test_norm_in_front_of_the_fused_output_layers(ctx):
    """runner.forward_lmhead with the models' last norms equals norms applied by hand, then the same call."""
    T, H, V = 40, 256, 2048
    g = torch.Generator(device="cuda").manual_seed(5)
    ha, hp = (torch.randn((T, H), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    wa, wp = ((torch.randn((V, H), generator=g, device="cuda") * 0.2).to(torch.bfloat16) for _ in range(2))
    tok = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    na = ((1 + 0.1 * torch.randn(H, generator=g, device="cuda")).to(torch.bfloat16), None, 1e-6, True)
    npol = (torch.ones(H, device="cuda"), torch.zeros(H, device="cuda") + 0.1, 1e-5, False)
    got = runner.forward_lmhead(ctx, ha, wa, hp, wp, tok, lam=1.5, k=8, seed=3, norm_actor=na, norm_policy=npol)
    ya = runner.layer_norm(ctx, ha, na[0], None, eps=1e-6, rms=True)[0]
    yp = runner.layer_norm(ctx, hp, npol[0], npol[1], eps=1e-5)[0]
    want = runner.forward_lmhead(ctx, ya, wa, yp, wp, tok, lam=1.5, k=8, seed=3)
    for n in ("accept", "weight", "logp_actor", "logp_policy", "topk_idx_actor", "z_approx"):
        assert torch.equal(got[n], want[n]), n
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = runner.forward_lmhead(ctx, ha, wa, hp, wp, tok, lam=1.5, k=8, seed=3, norm_actor=na, norm_policy=npol)
    assert torch.equal(again["weight"], want["weight"])


def test_refusals(ctx):
    x, dy, w, b = make(4, 64, torch.bfloat16, torch.bfloat16, True, seed=1)
    y, mean, rstd = runner.layer_norm(ctx, x, w, b)
    bad = [
        (lambda: runner.layer_norm(ctx, x.half(), w, b), "bfloat16 or float32"),
        (lambda: runner.layer_norm(ctx, x, w[:63], b), "weight"),
        (lambda: runner.layer_norm(ctx, x, w, b.float()), "bias"),
        (lambda: runner.layer_norm(ctx, x.t(), w, b), "contiguous rows"),
        (lambda: runner.layer_norm(ctx, x[:1].expand(4, 64), w, b), "overlap"),
        (lambda: runner.layer_norm(ctx, x, w, b, eps=-1.0), "eps"),
        (lambda: runner.layer_norm(ctx, x, w, b, eps=float("nan")), "eps"),
        (lambda: runner.layer_norm(ctx, x, w, b, out=y[:3]), "out"),
        (lambda: runner.layer_norm(ctx, x.cpu(), w, b), "context is on"),
        (lambda: runner.layer_norm_backward(ctx, dy.float(), x, w, mean, rstd), "dtype"),
        (lambda: runner.layer_norm_backward(ctx, dy, x, w, mean.double(), rstd), "mean"),
        (lambda: runner.layer_norm_backward(ctx, dy, x, w, mean, rstd[:3]), "rstd"),
    ]
    for call, text in bad:
        with pytest.raises(B.JackpotError, match=text):
            call()
    # the C entry's own checks
    d = B.jp_norm_desc(T=4, H=64, dtype=B.JP_BF16, param_dtype=B.JP_BF16)
    ws = torch.empty(B.jp_layer_norm_workspace_bytes(ctx, 4, 64, B.JP_BF16), dtype=torch.uint8, device="cuda")
    dw = torch.empty(64, device="cuda")
    with pytest.raises(B.JackpotError, match="workspace"):
        B.jp_layer_norm_backward(ctx, d, dy, x, w, mean, rstd, y, dw, None, ws[:-1])
    with pytest.raises(B.JackpotError, match="NULL"):
        B.jp_layer_norm_backward(ctx, d, dy, x, w, None, rstd, y, dw, None, ws)
    with pytest.raises(B.JackpotError, match="NULL"):
        B.jp_layer_norm_forward(ctx, d, x, None, None, y, None, None)
    for field, value in (("T", -1), ("H", 0), ("ld_x", 63), ("dtype", 2), ("param_dtype", 5), ("flags", 2)):
        e = B.jp_norm_desc(T=4, H=64, dtype=B.JP_BF16, param_dtype=B.JP_BF16)
        setattr(e, field, value)
        with pytest.raises(B.JackpotError):
            B.jp_layer_norm_forward(ctx, e, x, w, b, y, None, None)
    B.jp_layer_norm_forward(ctx, d, x, w, b, y, None, None)            # the context works as before
    torch.cuda.synchronize()


@pytest.mark.parametrize("T,H", [(5, 8200), (300, 13824), (160, 20011), (3, 8191 * 3)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wide_backward_does_not_depend_on_what_the_workspace_held(ctx, T, H, dtype):
    """Widths beyond the registers that are no multiple of the block's 1024 threads: the place of dbias[c] is emptied by the thread that
    adds to it.  Every call, on a workspace of NaN or of large numbers, gives the same bits."""
    x, dy, w, b = make(T, H, dtype, torch.float32, True, seed=T + H)
    _, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS)
    d = B.jp_norm_desc(T=T, H=H, dtype=B._dtype_code(x), param_dtype=B.JP_F32)
    need = B.jp_layer_norm_workspace_bytes(ctx, T, H, d.dtype)
    ws = torch.empty(need // 4, device="cuda")
    first = None
    for i in range(40):
        ws.fill_(float("nan") if i % 2 else 1e30)
        dx, dw, db = torch.empty_like(x), torch.empty(H, device="cuda"), torch.empty(H, device="cuda")
        B.jp_layer_norm_backward(ctx, d, dy, x, w, mean, rstd, dx, dw, db, ws.view(torch.uint8))
        if first is None:
            first = (dx, dw, db)
            check_backward(first, dy, x, w, mean, rstd, False)
        assert all(torch.equal(a, c) for a, c in zip(first, (dx, dw, db)))


def far_rows(T, H, dtype, seed):
    """Rows whose mean is 1000 (fp32) or 50 (bf16, which holds no more of their spread) standard deviations from zero."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    at, sigma = (2000.0, 2.0) if dtype is torch.float32 else (1000.0, 20.0)
    x = (torch.randn((T, H), generator=g, device="cuda") * sigma + at).to(dtype)
    dy = torch.randn((T, H), generator=g, device="cuda").to(dtype)
    w = 1 + 0.3 * torch.randn(H, generator=g, device="cuda")
    b = 0.2 * torch.randn(H, generator=g, device="cuda")
    return x, dy, w, b


@pytest.mark.parametrize("T", [40, 2000])
@pytest.mark.parametrize("H", [63, 768, 1283, 2047, 2048, 4096, 5112, 8192, 8200])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("apart", [False, True])
def test_rows_far_from_zero_keep_their_spread(ctx, T, H, dtype, apart):
    """xhat = (x - mean) rstd with the difference taken first, whichever kernel the row count and the width choose (``apart``: matrices
    at different offsets to 16 bytes).  From the mean and rstd of the call itself, xhat is off by 2 u (difference and product) and y by u of
    each of its two terms more: below 4 u of their magnitudes.  In the backward, mean and rstd are inputs: nothing in a bar grows with
    |mean|; a weight's sum of up to 124 terms (8200: 14 rows in memory, then the lines; fewer elsewhere) and its xhat stay below 128 u."""
    x, dy, w, b = far_rows(T, H, dtype, seed=T + H)
    if apart:
        flat = torch.empty(T * H + 1, device="cuda", dtype=dtype)
        xo = flat[1:].view(T, H)
        x = xo.copy_(x)
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS)
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    ref = xh * w.double() + b.double()
    mag = (xh * w.double()).abs() + b.double().abs()
    assert ((y.double() - ref).abs() <= HALF[dtype] * ref.abs() * (1 + 2.0 ** -8) + 4 * U * mag).all()
    dx, dw, db = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd)
    rdx, rdw, rdb, mag, magw, magb = plain_backward(dy, x, w, mean, rstd, False)
    assert ((dx.double() - rdx).abs() <= HALF[dtype] * rdx.abs() * (1 + 2.0 ** -8) + 64 * U * mag).all()
    assert ((dw.double() - rdw).abs() <= 128 * U * magw).all()
    assert ((db.double() - rdb).abs() <= 128 * U * magb).all()


@pytest.mark.parametrize("T", [40, 2000])
@pytest.mark.parametrize("H", [1024, 2048, 4096, 8192, 16384])
def test_rows_of_one_value_give_the_bias(ctx, T, H):
    """Sums of 2000 over a power of two of columns, and their mean, are exact; so x - mean is 0 whatever rstd is (1000 here)."""
    w, b = torch.rand(H, device="cuda") + 0.5, torch.rand(H, device="cuda")
    x = torch.full((T, H), 2000.0, device="cuda")
    y, mean, rstd = runner.layer_norm(ctx, x, w, b, eps=EPS)
    assert (mean == 2000).all() and torch.equal(y, b.expand(T, H))
    dy = torch.randn((T, H), device="cuda")
    dx, dw, db = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd)
    assert (dw == 0).all()


def test_tiny_rows_without_eps(ctx):
    """Rows of 2^-66 with eps 0: rstd is 2^66, whose square is beyond fp32; dx is rstd times numbers near 1 all the same."""
    T, H = 6, 1024
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.where(torch.rand((T, H), generator=g, device="cuda") < 0.5, -1.0, 1.0) * 2.0 ** -66
    dy, w = torch.randn((T, H), generator=g, device="cuda"), 1 + 0.3 * torch.randn(H, generator=g, device="cuda")
    for rms in (True, False):
        rstd = torch.full((T,), 2.0 ** 66, device="cuda")
        mean = None if rms else torch.zeros(T, device="cuda")
        got = runner.layer_norm_backward(ctx, dy, x, w, mean, rstd, rms=rms)
        check_backward(got, dy, x, w, torch.zeros(T, device="cuda"), rstd, rms)
