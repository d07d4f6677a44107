"""Kernels whose blocks stay for the whole call: their grids are what the GPU holds at once, as the driver's occupancy says for each captured launch.
Where a grid is larger, its last blocks start behind the others' whole share of rows."""
import pytest
import torch
from cuda.bindings import driver

from paper_2602_06107_b200 import binding as B
from paper_2602_06107_b200 import build as jp_build
from paper_2602_06107_b200 import runner

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    jp_build.build()
    c = B.Context(0)
    yield c
    c.close()


def answer(r):
    assert r[0] == driver.CUresult.CUDA_SUCCESS, r[0]
    return r[1] if len(r) == 2 else r[1:]


def launches(call, name):
    """(blocks, blocks that fit the GPU, blocks an SM, threads) of the kernels with that name in a captured call."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    g = driver.CUgraph(graph.raw_cuda_graph())
    nodes = answer(driver.cuGraphGetNodes(g, answer(driver.cuGraphGetNodes(g))[1]))[0]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    found = []
    for node in nodes:
        if answer(driver.cuGraphNodeGetType(node)) != driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            continue
        p = answer(driver.cuGraphKernelNodeGetParams(node))
        func = p.func if int(p.func) else answer(driver.cuKernelGetFunction(p.kern))
        if name not in answer(driver.cuFuncGetName(func)).decode():
            continue
        threads = p.blockDimX * p.blockDimY * p.blockDimZ
        each = answer(driver.cuOccupancyMaxActiveBlocksPerMultiprocessor(func, threads, p.sharedMemBytes))
        cluster = answer(driver.cuGraphKernelNodeGetAttribute(node, driver.CUlaunchAttributeID.CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION)).clusterDim.x or 1
        blocks = p.gridDimX * p.gridDimY * p.gridDimZ
        fit = each * sms
        if cluster > 1:
            attr = driver.CUlaunchAttribute()
            attr.id = driver.CUlaunchAttributeID.CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION
            attr.value.clusterDim.x, attr.value.clusterDim.y, attr.value.clusterDim.z = cluster, 1, 1
            cfg = driver.CUlaunchConfig()
            cfg.gridDimX, cfg.gridDimY, cfg.gridDimZ = blocks, 1, 1
            cfg.blockDimX, cfg.blockDimY, cfg.blockDimZ = threads, 1, 1
            cfg.sharedMemBytes, cfg.attrs, cfg.numAttrs = p.sharedMemBytes, [attr], 1
            fit = cluster * answer(driver.cuOccupancyMaxActiveClusters(func, cfg))
        found.append((blocks, fit, each, threads))
    assert found, name
    return found


def loss_call(ctx, T, V, dtype, grad):
    z = torch.zeros((T, (V + 7) // 8 * 8), device="cuda", dtype=dtype)[:, :V]
    tok, f = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.ones(T, device="cuda")
    return lambda: runner.policy_loss(ctx, z, tok, f, f, grad=grad)


# by vocabulary: vectors a thread up to the most, blocks a row from one to eight, 256 and 512 threads
LOSSES = [(700, 20011, BF), (700, 24000, BF), (700, 27000, BF), (700, 12000, F32), (700, 14000, F32), (700, 32000, BF), (700, 50257, BF), (700, 50257, F32),
          (400, 100277, BF), (300, 151936, BF), (300, 200064, BF), (160, 220000, BF), (160, 400000, BF), (4, 400000, BF), (3000, 1000, BF), (3000, 5003, F32)]


@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("T,V,dtype", LOSSES)
def test_rows_of_logits(ctx, T, V, dtype, grad):
    for blocks, fit, each, threads in launches(loss_call(ctx, T, V, dtype, grad), "loss_rows_kernel"):
        assert blocks <= fit, (blocks, fit, each, threads)


@pytest.mark.parametrize("T,V,dtype", [(700, 20011, BF), (700, 24000, BF), (700, 26624, BF), (700, 32000, BF), (700, 50257, BF), (700, 25000, F32), (700, 50257, F32),
                                       (400, 100277, BF), (300, 151936, BF), (300, 200064, BF), (300, 212992, BF), (300, 106496, F32)])
def test_four_blocks_an_sm(ctx, T, V, dtype):
    """Rows that 13 vectors a thread of up to eight blocks of 256 threads hold (fp32: of two blocks or more)."""
    for blocks, fit, each, threads in launches(loss_call(ctx, T, V, dtype, True), "loss_rows_kernel"):
        assert threads == 256 and each == 4 and blocks <= fit, (blocks, fit, each, threads)


def block_call(ctx, T, H, dtype, full, ld):
    m = lambda: torch.zeros((T, ld), device="cuda", dtype=dtype)[:, :H]
    x, r, y, total = m(), m(), m(), m()
    w = torch.ones(H, device="cuda")
    extra = dict(post_weight=w, gate=w, token_gate=torch.ones(T, device="cuda")) if full else dict(post_weight=w)

    def call():
        f = runner.block_norm(ctx, x, r, w, eps=1e-6, rms=not full, out=y, out_sum=total, **extra)
        runner.block_norm_backward(ctx, y, None, x, total, w, f["mean"], f["rstd"], post_mean=f["post_mean"], post_rstd=f["post_rstd"], rms=not full, bias=full, **extra)
    return call


# every number of threads a row from 32 to 1024, with 8 and 16 elements each; rows on 16 bytes and off them
@pytest.mark.parametrize("H", [8, 64, 256, 264, 500, 512, 520, 768, 1000, 1024, 1283, 1536, 2047, 2048, 2560, 4095, 4096, 5120, 8191, 8192, 16384])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("full", [True, False])
def test_rows_of_block_norms(ctx, H, dtype, full):
    for T in (300, 9600, 40000 if H <= 2048 else 9601):
        call = block_call(ctx, T, H, dtype, full, H)
        for name in ("block_fwd_kernel", "block_bwd_kernel") if H <= 5120 else ("block_fwd",):
            for blocks, fit, each, threads in launches(call, name):
                assert blocks <= fit, (name, T, blocks, fit, each, threads)
