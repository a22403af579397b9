"""Which launches the products' rules choose, on both sides of each, read from captured graphs; each result within the products' bound."""
import pytest
import torch

from tests import dense_oracle as orc
from tests.test_gpu_dense_runs import within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dense():
    from paper_2510_24061_b200 import dense
    return dense


def clusters(call):
    """CTAs of a cluster of each kernel launch that `call` makes, in their order, and the kernels' names."""
    from cuda.bindings import driver

    def ok(result):
        assert result[0] == driver.CUresult.CUDA_SUCCESS, result[0]
        return result[1] if len(result) == 2 else result[1:]

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        kept = call()  # noqa: F841
    raw = driver.CUgraph(graph.raw_cuda_graph())
    _, n = ok(driver.cuGraphGetNodes(raw))
    nodes, _ = ok(driver.cuGraphGetNodes(raw, n))
    out = []
    for node in nodes:
        if ok(driver.cuGraphNodeGetType(node)) != driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            continue
        p = ok(driver.cuGraphKernelNodeGetParams(node))
        name = ok(driver.cuKernelGetName(p.kern)) if int(p.kern) else ok(driver.cuFuncGetName(p.func))
        dim = ok(driver.cuGraphKernelNodeGetAttribute(node, driver.CUlaunchAttributeID.CU_LAUNCH_ATTRIBUTE_CLUSTER_DIMENSION)).clusterDim
        out.append((dim.x * dim.y * dim.z, name.decode()))
    return out


def random(rows, cols, seed):
    return torch.randn((rows, cols), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def operands(dense, way, T, n, m):
    """(call, its operands in 64 bits)"""
    if way == "dw":
        a, b = dense.block_quantize(random(T, m, 1), "col"), dense.block_quantize(random(T, n, 2), "col")
        return (lambda dtype=torch.float32: dense.block_weight_grad(a, b, dtype)), orc.value(a).T, orc.value(b)
    w = dense.block_quantize(random(m, n, 3), "tile")
    if way == "fwd":
        x = dense.block_quantize(random(T, n, 4))
        return (lambda dtype=torch.bfloat16: dense.block_forward(x, w, dtype)), orc.value(x), orc.value(w).T
    dy = dense.block_quantize(random(T, m, 5))
    return (lambda dtype=torch.bfloat16: dense.block_input_grad(dy, w, dtype)), orc.value(dy), orc.value(w)


@pytest.mark.parametrize("way,T,n,m,launches", [("dx", 777, 5120, 13824, 2), ("dx", 768, 5120, 13824, 1), ("fwd", 777, 13824, 5120, 2), ("fwd", 768, 13824, 5120, 1),
                                                ("dx", 1030, 4096, 11008, 2), ("dx", 1030, 4096, 4096, 1), ("fwd", 1030, 4096, 4096, 1), ("fwd", 300, 4096, 4096, 1)])
def test_rows_behind_whole_tiles(dense, way, T, n, m, launches):
    call, a, b = operands(dense, way, T, n, m)
    assert len(clusters(call)) == launches
    within(call(), a, b)
    within(call(torch.float32), a, b)


@pytest.mark.parametrize("way,T,n,m,size", [("dw", 16384, 1024, 256, 8), ("fwd", 8, 11008, 4096, 4), ("dw", 16384, 1024, 2048, 4), ("dw", 4096, 4096, 4096, 2),
                                            ("fwd", 512, 4096, 4096, 2), ("dw", 100, 1024, 256, 2)])
def test_clusters_that_share_a_tile(dense, way, T, n, m, size):
    """Few tiles and a long contraction: four pairs to a tile, or two where there are too many tiles for four; else one."""
    call, a, b = operands(dense, way, T, n, m)
    assert [c for c, _ in clusters(call)] == [size]
    for dtype in (torch.bfloat16, torch.float32):
        within(call(dtype), a, b)


@pytest.mark.parametrize("T,n,m,dtype,size,sums", [(8192, 1024, 256, torch.float32, 8, False), (8192 + 512, 1024, 256, torch.float32, 8, True),
                                                   (131072, 1024, 256, torch.bfloat16, 8, False), (2048, 4096, 4096, torch.float32, 2, False),
                                                   (2048 + 1, 4096, 4096, torch.float32, 2, True), (4096, 4096, 4096, torch.bfloat16, 2, False)])
def test_sums_of_several_parts(dense, T, n, m, dtype, size, sums):
    """fp32 results of more than 2048 terms a pair are summed in parts, by the kernel made for it."""
    call, _, _ = operands(dense, "dw", T, n, m)
    (got, name), = clusters(lambda: call(dtype))
    assert got == size and ("Lb1E" in name) == sums, (got, name)
