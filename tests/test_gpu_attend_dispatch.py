"""Which kernel attention takes: few tokens of many fp32 heads are not prompts."""

import ctypes

import pytest
import torch

from tests import attend_util as U

pytestmark = pytest.mark.gpu
D = 128


def kernels(call):
    """Names of the kernels that `call` launches, from a captured graph of it."""
    class Node(ctypes.Structure):                       # hipKernelNodeParams
        _fields_ = [("block", ctypes.c_uint * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3),
                    ("params", ctypes.c_void_p), ("shared", ctypes.c_uint)]

    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    hip = ctypes.CDLL(next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line))
    hip.hipKernelNameRefByPtr.restype = ctypes.c_char_p
    handle, count = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert hip.hipGraphGetNodes(handle, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(handle, nodes, ctypes.byref(count)) == 0
    names = []
    for node in nodes:
        p = Node()
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0
        names.append(hip.hipKernelNameRefByPtr(ctypes.c_void_p(p.func), None).decode())
    return names


@pytest.mark.parametrize("count,m,window,kernel", [(22, 1, 0, "split"), (32, 1, 300, "split"), (128, 1, 0, "split"), (32, 8, 0, "split"), (32, 64, 0, "prompt_f32"), (64, 17, 0, "prompt_f32")])
def test_fp32(count, m, window, kernel):
    n, kv = 600, 8
    K, V, Q = (U.randn(i, (count, kv if i < 3 else m, n if i < 3 else kv * 4, D), torch.float32) for i in (1, 2, 3))
    out, lse = torch.empty_like(Q), torch.empty((count, kv * 4, m), device="cuda")
    with U.context(kv, 4, "fp32", n) as ctx:
        call = lambda: ctx.attend(Q, K, V, count, m, n, n, out, window=window, n_sink=4, lse=lse)
        call()
        torch.cuda.synchronize()
        names = kernels(call)
    assert len(names) == 1 and f"attend_{kernel}_kernel" in names[0], names
    seen = U.causal(m, n, n, window, 4)
    for b, h in ((0, 0), (count - 1, 31)):
        U.check_attention(out[b, :, h], lse[b, h], U.attention(Q[b, :, h], K[b, h // 4], V[b, h // 4], seen, D ** -0.5), "fp32", n, f"seq {b} head {h}")
