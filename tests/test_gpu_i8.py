"""Linear layers in 8-bit integers (jp_i8_pack, jp_i8_quantize, jp_i8_linear) against exact integers.

Bars.  u = 2^-24.  The integers and their sums are exact, so the only errors are the scale of a token (one rounding, u), its product with the
channel's scale (u), the sum as fp32 (u) and their product (u): 4 u relative, below 4.01 u with their products, and the output's rounding: none more for fp32, half a step, 2^-8, for bf16."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def make(M, N, K, seed, ld_x=None, ld_q=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((M, ld_x or K), float("nan"), device="cuda", dtype=BF)
    x[:, :K] = (torch.randn((M, K), generator=g, device="cuda") * (1 + 5 * (torch.rand(K, generator=g, device="cuda") < 0.05))).to(BF)
    q = torch.full((N, ld_q or K), 77, device="cuda", dtype=torch.int8)
    q[:, :K] = torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    scales = (torch.rand(N, generator=g, device="cuda") + 0.5) * 0.01
    return x[:, :K], q[:, :K], scales


def rounded(x):
    """The tokens' integers and scales: in 64 bits the quotient of a half is a half, and nothing else is near one (see the kernel)."""
    x = x.double()
    most = x.abs().amax(1, keepdim=True)
    return torch.where(most > 0, 127 * x / most.clamp(min=1e-300), 0.0).round(), most / 127


def check(out, x, q, scales):
    xq, sx = rounded(x)
    want = torch.empty(out.shape, dtype=torch.float64, device="cuda")
    for n in range(0, q.shape[0], 4096):
        want[:, n:n + 4096] = (xq @ q[n:n + 4096].double().t()) * sx * scales[n:n + 4096].double()
    bar = (4.01 * U + (2.0 ** -8 if out.dtype is BF else 0)) * want.abs()
    assert ((out.double() - want).abs() <= bar).all()


MS = [1, 2, 7, 8, 9, 16, 17, 31, 33, 48, 63, 100, 127, 200, 256, 257, 300, 513, 777, 1025]


@pytest.mark.parametrize("M", MS)
@pytest.mark.parametrize("N,K", [(1, 1), (5, 15), (127, 16), (128, 100), (129, 127), (1000, 128), (300, 129), (640, 1111), (2048, 2048), (5003, 640)])
def test_sizes(ctx, M, N, K):
    x, q, scales = make(M, N, K, M * 1000 + N + K)
    w = runner.pack_i8(ctx, q, scales)
    for dtype in (BF, F32):
        out = runner.linear_i8(ctx, x, w, out_dtype=dtype)
        assert out.shape == (M, N)
        check(out, x, q, scales)
    assert torch.equal(runner.linear_i8(ctx, runner.quantize_tokens_i8(ctx, x), w, out_dtype=F32), out)


@pytest.mark.parametrize("M,N,K", [(1, 300, 65536), (40, 130, 65536), (300, 256, 16384), (3, 151936, 256), (48, 30000, 1024), (4100, 1300, 520), (70, 19000, 384),
                                   (600, 20000, 300), (1, 128, 8192), (20, 2048, 5120), (2500, 2500, 2500), (257, 37900, 129), (1000, 12801, 256), (129, 38000, 90),
                                   (513, 19999, 640), (4096, 4096, 384), (7777, 1500, 1111)])
def test_large_sizes(ctx, M, N, K):
    x, q, scales = make(M, N, K, M + N + K)
    w = runner.pack_i8(ctx, q, scales)
    out = runner.linear_i8(ctx, x, w, out_dtype=F32)
    check(out, x, q, scales)
    assert torch.equal(runner.linear_i8(ctx, x, w, out_dtype=F32), out)
    assert torch.equal(runner.linear_i8(ctx, x, w), out.to(BF))


@pytest.mark.parametrize("K", [64, 200, 1000, 5000])
def test_halves_go_to_the_even_integer(ctx, K):
    """Rows whose quotients are exact halves, next to halves, and everything else a bf16 can be, read back through a layer of single weights."""
    g = torch.Generator(device="cuda").manual_seed(K)
    M = 64
    x = torch.randn((M, K), generator=g, device="cuda")
    x[::2] = torch.randint(-254, 255, (M // 2, K), generator=g, device="cuda").float() / 2
    x[::2, 0] = 127.0                            # 127 x / max = x: every other one a half
    x[1::4, 1] = 200.0
    x = x.to(BF)
    x[2] = x[2] * 2.0 ** -126                    # near the smallest numbers, and subnormal ones
    x[4] = x[4] * 2.0 ** -133
    x[6] = x[6] * 2.0 ** 120
    x[8] = 0.0
    x[10] = 0.0
    x[10, K - 1] = 2.0 ** -133
    eye = torch.eye(K, dtype=torch.int8, device="cuda")
    out = runner.linear_i8(ctx, x, runner.pack_i8(ctx, eye, torch.ones(K, device="cuda")), out_dtype=F32)
    xq, sx = rounded(x)
    near = (xq * sx)
    # (a scale below 2^-126 is a multiple of 2^-149 only)
    assert ((out.double() - near).abs() <= 3 * U * near.abs() + xq.abs() * 2.0 ** -150).all()
    # the integers themselves, from rows that are scaled by powers of two
    back = (out / out.abs().amax(1, keepdim=True) * 127)[[0, 12, 14, 16]]
    assert ((back.double() - xq[[0, 12, 14, 16]]).abs() < 1e-3).all()


def test_tokens_without_numbers(ctx):
    x, q, scales = make(20, 200, 300, 3)
    x[3, 7], x[5, 0], x[9, 299] = float("nan"), float("inf"), float("-inf")
    x[11] = 0
    out = runner.linear_i8(ctx, x, runner.pack_i8(ctx, q, scales), out_dtype=F32)
    bad = [3, 5, 9]
    good = [i for i in range(20) if i not in bad]
    assert out[bad].isnan().all() and (out[11] == 0).all()
    check(out[good], x[good], q, scales)


@pytest.mark.parametrize("M,N,K,ld_x,ld_q", [(5, 100, 64, 65, 67), (33, 1000, 333, 336, 333), (300, 500, 1000, 1003, 1024), (1, 640, 256, 256, 256)])
def test_pitches_and_places(ctx, M, N, K, ld_x, ld_q):
    """Odd pitches and starts; out in a slice of wider rows, with nothing written beside it."""
    x, q, scales = make(M, N, K, 5, ld_x, ld_q)
    w = runner.pack_i8(ctx, q, scales)
    for dtype in (BF, F32):
        big = torch.full((M + 2, N + 5), 7.0, device="cuda", dtype=dtype)
        out = runner.linear_i8(ctx, x, w, out=big[1:M + 1, 3:3 + N])
        check(out, x, q, scales)
        assert (big[0] == 7).all() and (big[-1] == 7).all() and (big[:, :3] == 7).all() and (big[:, 3 + N:] == 7).all()
    flat = torch.empty(M * K + 1, dtype=BF, device="cuda")
    xo = flat[1:].view(M, K)
    xo.copy_(x)
    assert torch.equal(runner.linear_i8(ctx, xo, w, out_dtype=F32), runner.linear_i8(ctx, x, w, out_dtype=F32))


@pytest.mark.parametrize("N,K", [(7, 16384), (2048, 16384), (2048, 16385), (11840, 4096), (11848, 4096), (9001, 5009), (1024, 4096), (1025, 4097)])
def test_one_token(ctx, N, K):
    """One token, quantised in the same kernel up to some size: the same bits as in two steps, from any place of x."""
    x, q, scales = make(6, N, K, N + K, K + 3)
    x[3] = 0
    x[4, K - 1], x[5, 0] = float("nan"), float("-inf")
    w = runner.pack_i8(ctx, q, scales)
    for i in range(6):
        row = x[i:i + 1]
        out = runner.linear_i8(ctx, row, w, out_dtype=F32)
        two = runner.linear_i8(ctx, runner.quantize_tokens_i8(ctx, row), w, out_dtype=F32)
        assert torch.equal(out.view(torch.int32), two.view(torch.int32)) or (i > 3 and out.isnan().all() and two.isnan().all())
        if i < 4:
            check(out, row, q, scales)
            check(runner.linear_i8(ctx, row, w), row, q, scales)


def test_no_tokens(ctx):
    x, q, scales = make(4, 100, 64, 1)
    w = runner.pack_i8(ctx, q, scales)
    assert runner.linear_i8(ctx, x[:0], w).shape == (0, 100)
    t = runner.quantize_tokens_i8(ctx, x[:0])
    assert t.M == 0 and runner.linear_i8(ctx, t, w).shape == (0, 100)


def test_quantized_weights(ctx):
    """quantize_i8: off by half a step of the channel's scale at most."""
    g = torch.Generator(device="cuda").manual_seed(2)
    weight = torch.randn((300, 200), generator=g, device="cuda")
    weight[7] = 0
    q, scales = runner.quantize_i8(weight)
    assert q.dtype == torch.int8 and (q[7] == 0).all() and scales[7] == 0
    assert ((q.double() * scales.double()[:, None] - weight.double()).abs() <= scales.double()[:, None] * (0.5 + 200 * U)).all()
    x = torch.randn((6, 200), generator=g, device="cuda").to(BF)
    check(runner.linear_i8(ctx, x, runner.pack_i8(ctx, q, scales), out_dtype=F32), x, q, scales)


def test_offsets_beyond_32_bits(ctx):
    """An output of more than 2^31 elements, and weights of more than 2^32 bytes."""
    x, q, scales = make(17000, 130000, 128, 9)
    w = runner.pack_i8(ctx, q, scales)
    out = runner.linear_i8(ctx, x, w)
    for rows in (slice(0, 3), slice(16998, 17000)):
        check(out[rows], x[rows], q, scales)
    del out, w, q
    N, K = 70000, 65536
    q = torch.zeros((N, K), dtype=torch.int8, device="cuda")
    q[-3:] = torch.randint(-128, 128, (3, K), device="cuda", dtype=torch.int32).to(torch.int8)
    scales = torch.rand(N, device="cuda")
    w = runner.pack_i8(ctx, q, scales)
    x = torch.randn((2, K), device="cuda").to(BF)
    out = runner.linear_i8(ctx, x, w, out_dtype=F32)
    check(out[:, -3:], x, q[-3:], scales[-3:])
    assert (out[:, :-3] == 0).all()


def test_streams_graphs_and_layers_in_a_row(ctx):
    """A layer reads what the one in front wrote; two streams at once; graphs replayed with new inputs; weights laid out anew in between."""
    N, K = 1000, 512
    data = [make(m, N, K, m) for m in (40, 300)]
    second = make(1, 700, N, 4)
    w2 = runner.pack_i8(ctx, second[1], second[2])
    ws = [runner.pack_i8(ctx, q, s) for _, q, s in data]
    both = lambda i: runner.linear_i8(ctx, runner.linear_i8(ctx, data[i][0], ws[i]), w2, out_dtype=F32)
    want = [both(0), both(1)]
    for i in (0, 1):
        mid = runner.linear_i8(ctx, data[i][0], ws[i])
        check(want[i], mid, second[1], second[2])
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], []
    for i, st in enumerate(streams):
        with torch.cuda.stream(st):
            got.append(both(i))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs, outs = [], []
    for i in (0, 1):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(both(i))
        graphs.append(graph)
    fresh = [make(m, N, K, m + 1) for m in (40, 300)]
    for old, new in zip(data, fresh):
        old[0].copy_(new[0])
    for st, graph in zip(streams, graphs):
        with torch.cuda.stream(st):
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, both(i)) for i, a in enumerate(outs))
    t = runner.quantize_tokens_i8(ctx, data[0][0])
    for i in range(20):                          # the layer right behind the layout of its weights
        q = torch.roll(data[0][1], i, 0)
        w = runner.pack_i8(ctx, q, data[0][2])
        check(runner.linear_i8(ctx, t, w, out_dtype=F32), data[0][0], q, data[0][2])
        check(runner.linear_i8(ctx, data[0][0], runner.pack_i8(ctx, q, data[0][2]), out_dtype=F32), data[0][0], q, data[0][2])


def test_status_and_refusals(ctx):
    x, q, scales = make(4, 100, 64, 1)
    w = runner.pack_i8(ctx, q, scales)
    t = runner.quantize_tokens_i8(ctx, x)
    bad = [
        (lambda: runner.pack_i8(ctx, q.int(), scales), "int8"), (lambda: runner.pack_i8(ctx, q[0], scales), "int8 matrix"), (lambda: runner.pack_i8(ctx, q, scales[:9]), "scales"),
        (lambda: runner.pack_i8(ctx, q, scales.double()), "scales"), (lambda: runner.pack_i8(ctx, q.t(), scales[:64]), "contiguous rows"),
        (lambda: runner.pack_i8(ctx, torch.empty((1, 65537), dtype=torch.int8, device="cuda"), scales[:1].contiguous()), "no layout"),
        (lambda: runner.linear_i8(ctx, x.float(), w), "bfloat16"), (lambda: runner.linear_i8(ctx, x[:, :63], w), "63 columns"), (lambda: runner.linear_i8(ctx, x.t(), w), "contiguous rows"),
        (lambda: runner.linear_i8(ctx, x, w, out_dtype=torch.float16), "bfloat16 or float32"), (lambda: runner.linear_i8(ctx, x, w, out=torch.empty((3, 100), device="cuda")), "out must be"),
        (lambda: runner.linear_i8(ctx, x.cpu(), w), "context is on"), (lambda: runner.linear_i8(ctx, runner.I8Tokens(t.data, 4, 63), w), "63 columns"),
        (lambda: runner.linear_i8(ctx, runner.I8Tokens(t.data, 9, 64), w), "tokens is NULL or smaller"), (lambda: runner.quantize_tokens_i8(ctx, x[:, :0]), "0 columns"),
    ]
    for call, text in bad:
        with pytest.raises(B.JackpotError, match=text):
            call()
    # the C entry's own checks
    out, status = torch.empty((4, 100), device="cuda"), torch.full((1,), 5, dtype=torch.int32, device="cuda")
    call = lambda desc=w.desc, packed=w.packed, xx=x, ld_x=64, M=4, tok=t.data, oo=out, ld=100, dt=B.JP_F32: B.jp_i8_linear(ctx, desc, packed, xx, ld_x, M, tok, oo, ld, dt, status)
    for k, text in ((dict(desc=B.jp_i8_desc(N=0, K=64)), "N out"), (dict(desc=B.jp_i8_desc(N=100, K=65537)), "K out"), (dict(M=-1), "M < 0"), (dict(M=1 << 24), "2\\^24"), (dict(ld_x=63), "leading"),
                    (dict(ld=99), "leading"), (dict(dt=2), "out must be"), (dict(packed=None), "NULL"), (dict(oo=None), "NULL"), (dict(tok=t.data[:100]), "jp_i8_token_bytes"),
                    (dict(tok=t.data[1:]), "jp_i8_token_bytes|aligned"), (dict(packed=w.packed[1:]), "16-byte")):
        with pytest.raises(B.JackpotError, match=text):
            call(**k)
    call()
    assert status.item() == 0
    check(out, x, q, scales)


@pytest.mark.parametrize("M", [1, 5])
def test_out_in_the_place_of_x_is_refused(ctx, M):
    x, q, scales = make(M, 64, 64, 2)
    with pytest.raises(B.JackpotError, match="the same matrix"):
        runner.linear_i8(ctx, x, runner.pack_i8(ctx, q, scales), out=x)
