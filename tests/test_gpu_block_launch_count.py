"""The launch count of a model with gated blocks against the kernel nodes of a captured step: what a block's calls consist of depends on precision, widths and
rows (contractions with split sums and copies into padded rows in float and at odd widths, one or two launches for a backward pass's products)."""
import ctypes

import pytest

import sb_inputs as si

from test_gpu_gated_block import GATED, batch, device, make_params, model, sb, workload


def kernel_nodes(graph):
    cuda = ctypes.CDLL("libcuda.so.1")
    handle, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert cuda.cuGraphGetNodes(handle, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert cuda.cuGraphGetNodes(handle, nodes, ctypes.byref(n)) == 0
    kinds = []
    for node in nodes:
        kind = ctypes.c_int(-1)
        assert cuda.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        kinds.append(kind.value)
    return kinds.count(0)          # CU_GRAPH_NODE_TYPE_KERNEL


@pytest.mark.gpu
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("width,hidden,b", [(64, (96, 40), 4), (33, (45,), 4), (128, (264,), 300)])
def test_launch_count_is_the_number_of_kernels(bf16, width, hidden, b):
    import torch
    lib = sb()
    layers = [(si.FC_RELU, width), *[(GATED, f) for f in hidden], (si.FC, 10), (si.SOFTMAX_XENT, 10)]
    wl = workload([(si.CONV3X3_RELU, 8), (si.MAXPOOL2, 0)] + layers, b=b)
    m = model(lib, wl, make_params(wl), lib.SB_BF16 if bf16 else lib.SB_FP32, lib.SB_FLAG_ADAMW)
    xs, ys = device(wl, *batch(wl, 0), bf16)

    def step():
        m.forward(xs, ys)
        m.backward()
        m.adamw_step(1e-3, step=1)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph(keep_graph=True)
        with torch.cuda.graph(graph, stream=stream):
            step()
        counted, launched = m.launch_count(), kernel_nodes(graph)
    torch.cuda.synchronize()
    m.close()
    assert counted == launched
