"""The kernels that a call launches, as a captured graph holds them."""

import ctypes

import torch


class _KernelNode(ctypes.Structure):
    """The driver's parameters of a kernel node."""
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3),
                ("smem", ctypes.c_uint), ("params", ctypes.c_void_p), ("extra", ctypes.c_void_p),
                ("kernel", ctypes.c_void_p), ("context", ctypes.c_void_p)]


def kernels(call):
    """The (mangled) names of the kernels that call() launches, which runs once before it is captured."""
    driver = ctypes.CDLL("libcuda.so.1")

    def ok(code):
        assert code == 0, code

    call()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    ok(driver.cuGraphGetNodes(raw, None, ctypes.byref(n)))
    nodes = (ctypes.c_void_p * n.value)()
    ok(driver.cuGraphGetNodes(raw, nodes, ctypes.byref(n)))
    names = []
    for node in nodes:
        kind, p, name = ctypes.c_int(), _KernelNode(), ctypes.c_char_p()
        ok(driver.cuGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)))
        if kind.value:  # (0: a kernel)
            continue
        ok(driver.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(p)))
        ok(driver.cuFuncGetName(ctypes.byref(name), ctypes.c_void_p(p.func)) if p.func
           else driver.cuKernelGetName(ctypes.byref(name), ctypes.c_void_p(p.kernel)))
        names.append(name.value.decode())
    return names
