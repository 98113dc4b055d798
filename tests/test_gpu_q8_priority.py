"""The 8-bit operators run at the priority of the stream that they are called on."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    import paper_2506_16235_b200 as nsml

KERNEL_NODE, PRIORITY = 0, 8  # CU_GRAPH_NODE_TYPE_KERNEL, CU_LAUNCH_ATTRIBUTE_PRIORITY


def kernel_priorities(graph):
    """The launch priority of every kernel in a captured graph."""
    cuda, handle, count = ctypes.CDLL("libcuda.so.1"), ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert cuda.cuGraphGetNodes(handle, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert cuda.cuGraphGetNodes(handle, nodes, ctypes.byref(count)) == 0
    found = []
    for node in nodes:
        kind, value = ctypes.c_int(-1), (ctypes.c_int * 16)()  # (a union of 64 bytes)
        assert cuda.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value == KERNEL_NODE:
            assert cuda.cuGraphKernelNodeGetAttribute(ctypes.c_void_p(node), PRIORITY, value) == 0
            found.append(value[0])
    return found


@pytest.mark.parametrize("priority", [0, -1, -3])
def test_every_kernel_has_the_streams_priority(priority):
    m, n, k = 300, 264, 520
    x, w = torch.randn(m, k, device="cuda"), torch.randn(n, k, device="cuda")
    dy, weight = torch.randn(m, n, device="cuda").bfloat16(), torch.ones(k, device="cuda")
    stream = torch.cuda.Stream(priority=priority)

    def step():
        codes, scales, rstd, h = nsml.nsml_q8_rms_norm(x, weight)
        b, sb = nsml.nsml_q8_pack(w)
        nsml.nsml_q8_matmul(codes, scales, b, sb)
        nsml.nsml_q8_matmul(codes[:1], scales[:1], b, sb)
        nsml.nsml_q8_matmul_grad_weight(dy, codes, scales)
        dx = nsml.nsml_q8_matmul_grad_input(dy, b, sb, dtype=torch.float32)
        nsml.nsml_q8_rms_norm_backward(dx, weight, rstd, h=h)
        nsml.nsml_q8_unpack(codes, scales)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph, stream=stream):
        x.mul_(1.0)  # an ordinary kernel: it has the stream's priority
        step()
    found = kernel_priorities(graph)
    assert len(found) == 10 and found == [stream.priority] * 10
