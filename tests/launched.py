"""Which kernels a call launches, read from a graph that it is captured into and that never runs.  Not a test module."""
import torch


def kernels(call):
    """Names of the kernels that `call` launches, in order; everything that it copies or allocates has to be there before."""
    from cuda.bindings import driver

    def got(answer):
        assert answer[0] == driver.CUresult.CUDA_SUCCESS, answer[0]
        return answer[1] if len(answer) == 2 else answer[1:]

    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        call()
    raw = driver.CUgraph(graph.raw_cuda_graph())
    count = got(driver.cuGraphGetNodes(raw, 0))[1]
    names = []
    for node in got(driver.cuGraphGetNodes(raw, count))[0]:
        if got(driver.cuGraphNodeGetType(node)) == driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            names.append(got(driver.cuFuncGetName(got(driver.cuGraphKernelNodeGetParams(node)).func)).decode())
    return names
