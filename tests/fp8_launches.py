"""Which kernels a call launches: captured into a graph, and read from its nodes."""
import re

import torch
from cuda.bindings import driver


def _done(result):
    assert result[0] == driver.CUresult.CUDA_SUCCESS, result[0]
    return result[1] if len(result) == 2 else result[1:]


def launches(call):
    """[(name, template arguments, thread blocks across, down)] of a call, by name; the call is made once before."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        kept = call()
    raw = driver.CUgraph(graph.raw_cuda_graph())
    count = _done(driver.cuGraphGetNodes(raw, 0))[1]
    nodes = _done(driver.cuGraphGetNodes(raw, count))[0]
    found = []
    for node in nodes:
        assert _done(driver.cuGraphNodeGetType(node)) == driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL
        p = _done(driver.cuGraphKernelNodeGetParams(node))
        name = _done(driver.cuFuncGetName(p.func) if int(p.func) else driver.cuKernelGetName(p.kern)).decode()
        base = re.search(r"\d+([a-z_]+_kernel)I(.*?)E?Ev", name)
        args = re.findall(r"L[ib](\d+)E|(f)E|(__nv_bfloat16)", base.group(2) + "E")
        found.append((base.group(1), tuple(int(a) if a else ("f32" if f else "bf16") for a, f, b in args), p.gridDimX, p.gridDimY))
    del kept
    return sorted(found)
