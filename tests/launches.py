"""The kernels that a call launches, read from a captured graph: names and grids, without running them."""
import torch


def launched(call):
    """[(kernel name, CTAs, threads)] of the kernel launches that `call` makes on the current stream, in their order."""
    from cuda.bindings import driver

    def ok(result):
        assert result[0] == driver.CUresult.CUDA_SUCCESS, result[0]
        return result[1] if len(result) == 2 else result[1:]

    call()                                           # whatever a first call sets up
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
        out.append((name.decode(), p.gridDimX * p.gridDimY * p.gridDimZ, p.blockDimX))
    return out
