"""What a call launches, read from a graph that it was captured into (which is not replayed)."""
import ctypes
import re

import torch


class _Dim3(ctypes.Structure):
    _fields_ = [("x", ctypes.c_uint32), ("y", ctypes.c_uint32), ("z", ctypes.c_uint32)]


class _KernelNodeParams(ctypes.Structure):
    _fields_ = [("block", _Dim3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", _Dim3), ("params", ctypes.c_void_p),
                ("shared", ctypes.c_uint32)]


def _runtime():
    """The HIP runtime that the process has loaded."""
    with open("/proc/self/maps") as maps:
        paths = sorted(set(re.findall(r"\S*/libamdhip64\.so\S*", maps.read())))
    assert len(paths) == 1, paths
    return ctypes.CDLL(paths[0])


def launches(call):
    """[(workgroups, threads of each)] of the kernels that call() launches."""
    graph, side = torch.cuda.CUDAGraph(keep_graph=True), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    hip, raw = _runtime(), ctypes.c_void_p(graph.raw_cuda_graph())
    n = ctypes.c_size_t()
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(n)) == 0
    out = []
    for node in nodes:
        kind = ctypes.c_int()
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0
        if kind.value == 0:                                    # a kernel
            p = _KernelNodeParams()
            assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0
            out.append((p.grid.x * p.grid.y * p.grid.z, p.block.x * p.block.y * p.block.z))
    return out
