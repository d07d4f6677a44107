"""Linear layers with 4-bit weights (jp_w4_pack, jp_w4_linear) against a plain product in 64 bits.

Bar.  q - z and x are exact in bf16, so every product is exact and the error is that of fp32 sums.  u = 2^-24.  A group
of g columns is g / 16 tensor-core steps of 16 products; each step may truncate (2 u) and its tree of 16 adds up to four
levels, so at most 2 (8 + 4) u of the group's sum of magnitudes; then K / g scaled sums and up to 16 warps' parts are added (u
each), the scaling itself 2 u.  In all (48 + K / g) u sum |x| |w|, plus half a step of the output's type, 2^-8 relative for
bf16."""
import pytest
import torch

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

U = 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def make(N, K, group, zeros, scales, seed, dev="cuda"):
    g = torch.Generator(device=dev).manual_seed(seed)
    G = (K + group - 1) // group
    q = torch.randint(0, 256, (N, (K + 1) // 2), generator=g, device=dev, dtype=torch.int32).to(torch.uint8)
    s = ((torch.rand((N, G), generator=g, device=dev) + 0.1) * 0.02).to(scales)
    s[:, 0] *= -1                                           # a negative scale is a scale
    z = torch.randint(0, 16, (N, G), generator=g, device=dev, dtype=torch.int32).to(torch.uint8) if zeros else None
    return q, s, z


def unpacked(q, s, z, K, group):
    v = torch.stack([q & 15, q >> 4], 2).reshape(q.shape[0], -1)[:, :K].double()
    grp = torch.arange(K, device=q.device) // group
    return (v - (8.0 if z is None else z.double()[:, grp])) * s.double()[:, grp]


def tokens(M, K, seed, ld=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((M, ld or K), float("nan"), device="cuda", dtype=torch.bfloat16)
    x[:, :K] = (torch.randn((M, K), generator=g, device="cuda") * 3).to(torch.bfloat16)
    return x[:, :K]


def check(out, x, w, group):
    K = w.shape[1]
    ref = x.double() @ w.t()
    bar = (48 + K / group) * U * (x.double().abs() @ w.abs().t())
    if out.dtype == torch.bfloat16:
        bar = bar + 2.0 ** -8 * ref.abs()
    assert ((out.double() - ref).abs() <= bar).all(), float(((out.double() - ref).abs() / bar).max())


SIZES = [(1, 1), (1, 7), (16, 128), (17, 129), (5, 64), (40, 300), (333, 1111), (2048, 2048), (2500, 640), (64, 8192),
         (16, 65536), (5003, 257)]


@gpu
@pytest.mark.parametrize("N,K", SIZES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros,scales", [(False, torch.bfloat16), (True, torch.float16)])
def test_product_matches_the_formula(ctx, N, K, group, zeros, scales):
    q, s, z = make(N, K, group, zeros, scales, seed=N + K)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    ref = unpacked(q, s, z, K, group)
    for i, M in enumerate((1, 3, 8, 9, 16, 17, 32)):
        x = tokens(M, K, seed=M)
        out = runner.linear_w4(ctx, x, w, out_dtype=(torch.float32, torch.bfloat16)[i % 2])
        assert out.shape == (M, N)
        check(out, x, ref, group)


@gpu
@pytest.mark.parametrize("M", [1, 5, 20])
def test_output_layer_size(ctx, M):
    """A vocabulary of 151,936 rows: every SM holds many tiles, and warps share most of them."""
    N, K, group = 151936, 1024, 64
    q, s, z = make(N, K, group, True, torch.bfloat16, seed=2)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    x = tokens(M, K, seed=1)
    check(runner.linear_w4(ctx, x, w, out_dtype=torch.float32), x, unpacked(q, s, z, K, group), group)


@gpu
def test_exact_values(ctx):
    """Small integers and scales that are powers of two leave no rounding: results are equal, bit for bit."""
    N, K, group = 100, 384, 32
    q, _, z = make(N, K, group, True, torch.float16, seed=8)
    s = torch.full((N, K // group), 0.25, dtype=torch.float16, device="cuda")
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    x = torch.randint(-4, 5, (11, K), device="cuda").to(torch.bfloat16)
    out = runner.linear_w4(ctx, x, w, out_dtype=torch.float32)
    assert torch.equal(out.double(), x.double() @ unpacked(q, s, z, K, group).t())
    one = torch.zeros((1, K), device="cuda", dtype=torch.bfloat16)
    one[0, 200] = 1
    assert torch.equal(runner.linear_w4(ctx, one, w, out_dtype=torch.float32)[0].double(), unpacked(q, s, z, K, group)[:, 200])


@gpu
def test_pitches_and_what_lies_beside_the_output(ctx):
    N, K, group, M = 203, 333, 64, 9
    qf, sf, zf = make(N, K + 60, group, True, torch.bfloat16, seed=3)
    q, s, z = qf[:, :(K + 1) // 2], sf[:, :6], zf[:, :6]          # rows further apart than they are long
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    ref = unpacked(q, s, z, K, group)
    x = tokens(M, K, seed=4, ld=K + 11)                            # NaN beside the rows
    for dtype in (torch.float32, torch.bfloat16):
        big = torch.full((M + 2, N + 5), 3.0, device="cuda", dtype=dtype)
        out = runner.linear_w4(ctx, x, w, out=big[1:M + 1, 2:N + 2])
        check(out, x, ref, group)
        assert (big[0] == 3).all() and (big[-1] == 3).all() and (big[:, :2] == 3).all() and (big[:, N + 2:] == 3).all()
    odd = torch.empty(M * K + 1, dtype=torch.bfloat16, device="cuda")[1:].view(M, K)
    odd.copy_(x)
    assert torch.equal(runner.linear_w4(ctx, odd, w), runner.linear_w4(ctx, x, w))


@gpu
def test_tokens_are_independent(ctx):
    """A token of NaN or infinities leaves the others as they are; a token alone gives what it gives in a batch."""
    q, s, z = make(500, 512, 128, True, torch.bfloat16, seed=5)
    w = runner.pack_w4(ctx, q, s, z, K=512)
    x = tokens(12, 512, seed=6)
    clean = runner.linear_w4(ctx, x, w, out_dtype=torch.float32)
    x[3], x[7] = float("nan"), float("inf")
    out = runner.linear_w4(ctx, x, w, out_dtype=torch.float32)
    keep = [i for i in range(12) if i not in (3, 7)]
    assert torch.equal(out[keep], clean[keep]) and out[3].isnan().all() and not out[7].isfinite().any()
    for i in (0, 11):
        assert torch.equal(runner.linear_w4(ctx, x[i:i + 1], w, out_dtype=torch.float32)[0], clean[i])


@gpu
def test_no_tokens_and_streams_and_graphs(ctx):
    q, s, z = make(700, 1000, 64, False, torch.float16, seed=7)
    w = runner.pack_w4(ctx, q, s, z, K=1000, group=64)
    assert runner.linear_w4(ctx, torch.empty((0, 1000), dtype=torch.bfloat16, device="cuda"), w).shape == (0, 700)
    x = tokens(6, 1000, seed=8)
    first = runner.linear_w4(ctx, x, w)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = runner.linear_w4(ctx, x, w)
    side.synchronize()
    assert torch.equal(first, second)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = runner.linear_w4(ctx, x, w)
    x.copy_(x.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(third, first.flip(0))


@gpu
def test_refusals(ctx):
    q, s, z = make(20, 96, 32, True, torch.bfloat16, seed=1)
    w = runner.pack_w4(ctx, q, s, z, K=96, group=32)
    x = tokens(4, 96, seed=1)
    bad = [
        (lambda: runner.pack_w4(ctx, q, s, z, K=96, group=16), "group"),
        (lambda: runner.pack_w4(ctx, q, s, z, K=98, group=32), "q must be"),
        (lambda: runner.pack_w4(ctx, q, s[:, :2], z, K=96, group=32), "scales"),
        (lambda: runner.pack_w4(ctx, q, s, z[:19], K=96, group=32), "zeros"),
        (lambda: runner.pack_w4(ctx, q, s.float(), z, K=96, group=32), "scales bfloat16"),
        (lambda: runner.pack_w4(ctx, q.int(), s, z, K=96, group=32), "uint8"),
        (lambda: runner.pack_w4(ctx, q.cpu(), s, z, K=96, group=32), "context is on"),
        (lambda: runner.linear_w4(ctx, x.float(), w), "bfloat16"),
        (lambda: runner.linear_w4(ctx, x[:, :95], w), "columns"),
        (lambda: runner.linear_w4(ctx, tokens(33, 96, seed=1), w), "JP_W4_MAX_TOKENS"),
        (lambda: runner.linear_w4(ctx, x, w, out_dtype=torch.float16), "bfloat16 or float32"),
        (lambda: runner.linear_w4(ctx, x, w, out=torch.empty((4, 19), device="cuda")), "out must be"),
        (lambda: runner.linear_w4(ctx, x.t().contiguous().t(), w), "contiguous rows"),
    ]
    for call, text in bad:
        with pytest.raises(B.JackpotError, match=text):
            call()
    out = torch.empty((4, 20), device="cuda")
    for field, value in (("N", 0), ("K", 65537), ("group", 48)):
        d = B.jp_w4_desc(N=20, K=96, group=32)
        setattr(d, field, value)
        with pytest.raises(B.JackpotError):
            B.jp_w4_linear(ctx, d, w.packed, x, 96, 4, out, 20, B.JP_F32)
    for args in ((None, x, 96, 4, out, 20, B.JP_F32), (w.packed, x, 95, 4, out, 20, B.JP_F32),
                 (w.packed, x, 96, 4, out, 19, B.JP_F32), (w.packed, x, 96, -1, out, 20, B.JP_F32),
                 (w.packed[1:], x, 96, 4, out, 20, B.JP_F32), (w.packed, x, 96, 4, out, 20, B.JP_F16)):
        with pytest.raises(B.JackpotError):
            B.jp_w4_linear(ctx, w.desc, *args)
    check(runner.linear_w4(ctx, x, w, out_dtype=torch.float32), x, unpacked(q, s, z, 96, 32), 32)


def test_layout_size_on_the_host():
    jp_build.build()
    assert B.jp_w4_packed_bytes(16, 128, 128) == 1024 + 64
    assert B.jp_w4_packed_bytes(17, 129, 32) == 4 * (1024 + 256)
    assert B.jp_w4_packed_bytes(151936, 4096, 64) == 9496 * 32 * (1024 + 128)
    for bad in ((0, 128, 128), (16, 0, 128), (16, 128, 100), (16, 65537, 128), (2**31, 128, 128)):
        assert B.jp_w4_packed_bytes(*bad) == 0


@pytest.mark.parametrize("K,group", [(256, 128), (100, 32), (33, 64), (1, 32), (64, 64)])
@pytest.mark.parametrize("symmetric", [True, False])
def test_quantised_weights_are_within_half_a_step(K, group, symmetric):
    torch.manual_seed(K)
    w = torch.randn((9, K))
    w[2] = 0
    q, s, z = runner.quantize_w4(w, group, symmetric=symmetric)
    assert (z is None) == symmetric and q.shape == (9, (K + 1) // 2) and q.dtype == torch.uint8
    back = unpacked(q, s, z, K, group)
    step = s.double().abs()[:, torch.arange(K) // group]
    # half a step; the scale's rounding to bf16 (2^-8) can push the largest of 7 (15) steps out by 15 / 256 of one, the
    # rounded zero point of an uneven range by another half
    assert ((back - w.double()).abs() <= step * (0.5 + 15 / 256 + (0 if symmetric else 0.5)) + 1e-12).all()
    assert (back[2] == 0).all()


@gpu
@pytest.mark.parametrize("power,x_power", [(124, -20), (-120, 0)])
def test_scales_near_the_ends_of_bf16(ctx, power, x_power):
    """Weights up to 8 x 2^125 with small x, and down to 2^-121: neither the sums nor the scaled parts leave fp32.  (What a
    subnormal part loses is 2^-150 a group, far below the bar of 48 x 2^-24 of sums near 2^-112.)"""
    N, K, group = 70, 600, 32
    q, s, z = make(N, K, group, True, torch.bfloat16, seed=12)
    s = (s.double().sign() * (1 + s.double().abs()) * 2.0 ** power).to(torch.bfloat16)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    x = (tokens(6, K, seed=3).float() * 2.0 ** x_power).to(torch.bfloat16)
    check(runner.linear_w4(ctx, x, w, out_dtype=torch.float32), x, unpacked(q, s, z, K, group), group)


@gpu
@pytest.mark.parametrize("start", [0, 1, 2, 4, 8])
@pytest.mark.parametrize("M,ld", [(1, 0), (1, 601), (2, 600), (3, 601), (4, 604), (6, 601), (9, 608), (32, 603)])
def test_where_tokens_start(ctx, start, M, ld):
    """Rows of x on 16 bytes, 8, 4 and 2, alone and at any pitch; what is around them is NaN and is not read."""
    N, K, group = 50, 599, 64
    q, s, z = make(N, K, group, True, torch.bfloat16, seed=4)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    ld = ld or K
    flat = torch.full((start + M * ld,), float("nan"), device="cuda", dtype=torch.bfloat16)
    x = flat[start:].as_strided((M, K), (ld, 1), start)
    x.copy_(tokens(M, K, seed=M))
    check(runner.linear_w4(ctx, x, w, out_dtype=torch.float32), x, unpacked(q, s, z, K, group), group)


@gpu
@pytest.mark.parametrize("N,K", [(19000, 200), (18960, 1024), (18961, 129), (37900, 385)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_pairs_of_tiles(ctx, N, K, group):
    """Enough tiles that they are taken in pairs, an even and an odd number of them, with a short last one."""
    q, s, z = make(N, K, group, True, torch.float16, seed=N)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    ref = unpacked(q, s, z, K, group)
    for M in (1, 5, 8, 11):
        big = torch.full((M + 2, N + 3), 7.0, device="cuda")
        x = tokens(M, K, seed=M)
        out = runner.linear_w4(ctx, x, w, out=big[1:M + 1, :N])
        check(out, x, ref, group)
        assert (big[0] == 7).all() and (big[-1] == 7).all() and (big[:, N:] == 7).all()
        assert torch.equal(runner.linear_w4(ctx, x, w, out_dtype=torch.float32), out)


@gpu
@pytest.mark.parametrize("N,K,M", [(109, 6274, 28), (292, 2447, 32), (9217, 8126, 30), (1, 40000, 2), (16, 65536, 9), (700, 1100, 1),
                                   (4000, 8192, 13), (33, 3000, 7)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_columns_split_over_a_cluster(ctx, N, K, M, group):
    """Few rows with many columns, and more tokens than one block's shared memory holds; the same call gives the same bits."""
    q, s, z = make(N, K, group, True, torch.bfloat16, seed=K)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=group)
    big = torch.full((M + 2, N + 3), 7.0, device="cuda")
    x = tokens(M, K, seed=M)
    out = runner.linear_w4(ctx, x, w, out=big[1:M + 1, :N])
    check(out, x, unpacked(q, s, z, K, group), group)
    assert (big[0] == 7).all() and (big[-1] == 7).all() and (big[:, N:] == 7).all()
    assert torch.equal(runner.linear_w4(ctx, x, w, out_dtype=torch.float32), out)


@gpu
@pytest.mark.parametrize("N,K,M", [(109, 6274, 28), (19000, 300, 3), (9217, 4100, 32)])
def test_every_kind_of_launch_in_graphs_on_two_streams(ctx, N, K, M):
    """A captured call reads its inputs anew, and two of them may run at the same time."""
    q, s, z = make(N, K, 64, True, torch.bfloat16, seed=N)
    w = runner.pack_w4(ctx, q, s, z, K=K, group=64)
    xs, outs, graphs, streams = [], [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for i in range(2):
        xs.append(tokens(M, K, seed=i).clone())
        runner.linear_w4(ctx, xs[i], w)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(runner.linear_w4(ctx, xs[i], w, out_dtype=torch.float32))
        graphs.append(g)
    for again in range(3):
        for i in range(2):
            xs[i].copy_(tokens(M, K, seed=10 * again + i))
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], runner.linear_w4(ctx, xs[i], w, out_dtype=torch.float32))


@gpu
@pytest.mark.parametrize("N,K,M,launches", [(8192, 28672, 32, 2), (16, 65536, 32, 4), (18000, 8192, 32, 2), (4096, 14336, 32, 2), (2048, 2048, 32, 1),
                                            (42785, 6806, 30, 2), (40, 65536, 1, 1)])
def test_few_launches_where_x_does_not_fit(ctx, N, K, M, launches):
    """Every launch reads all weights: as many tokens in each as fit one block or a cluster of blocks."""
    q, s, z = make(N, K, 128, True, torch.bfloat16, seed=N)
    w = runner.pack_w4(ctx, q, s, z, K=K)
    x = tokens(M, K, seed=M)
    before = ctx.launch_count()
    out = runner.linear_w4(ctx, x, w, out_dtype=torch.float32)
    assert ctx.launch_count() - before == launches
    ref = unpacked(q, s, z, K, 128)
    check(out, x, ref, 128)
