"""Which of the library's kernels a call launches: captured into a graph whose nodes are then read by name.  For tests that want
to know that a size still takes the path it was chosen for."""
import re

import torch


def _ok(result):
    assert int(result[0]) == 0, result[0]
    return result[1:] if len(result) > 2 else result[1]


def kernels(call):
    """Names of the k_* kernels in the order of the graph's nodes; `call` is made once outside the graph and once in it."""
    from cuda.bindings import driver as cu
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw = cu.CUgraph(graph.raw_cuda_graph())
    nodes, count = _ok(cu.cuGraphGetNodes(raw))
    nodes, count = _ok(cu.cuGraphGetNodes(raw, count))
    names = []
    for node in nodes[:count]:
        if _ok(cu.cuGraphNodeGetType(node)) == cu.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            p = _ok(cu.cuGraphKernelNodeGetParams(node))
            name = _ok(cu.cuFuncGetName(p.func)) if int(p.func) else _ok(cu.cuKernelGetName(p.kern))
            names += re.findall(r"\d+(k_[a-z_]+)", name.decode())
    return names
