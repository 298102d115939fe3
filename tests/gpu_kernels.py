"""Which kernels a call launches, for tests that are meant to reach a particular one: the call is recorded into a graph, whose nodes are read and which never runs."""
import ctypes as C

import torch

import paper_2111_01264_amd as P

_LIB = C.CDLL(P.LIB_PATH)   # (symbols of the runtime that the library is linked to are found through it)
_RELAXED = 2


class _Dim3(C.Structure):
    _fields_ = [("x", C.c_uint32), ("y", C.c_uint32), ("z", C.c_uint32)]


class _KernelNode(C.Structure):
    _fields_ = [("block", _Dim3), ("extra", C.c_void_p), ("func", C.c_void_p), ("grid", _Dim3), ("params", C.c_void_p), ("lds", C.c_uint)]


def _ok(rc):
    assert rc == 0, "HIP error %d" % rc


def kernels_of(call):
    """Mangled names of the kernels that call(stream) launches, in order; every node of its graph is a kernel."""
    stream = torch.cuda.Stream()
    handle, graph, n = C.c_void_p(stream.cuda_stream), C.c_void_p(), C.c_size_t()
    torch.cuda.synchronize()
    _ok(_LIB.hipStreamBeginCapture(handle, _RELAXED))
    try:
        call(stream)
    finally:
        _ok(_LIB.hipStreamEndCapture(handle, C.byref(graph)))
    _ok(_LIB.hipGraphGetNodes(graph, None, C.byref(n)))
    nodes = (C.c_void_p * n.value)()
    _ok(_LIB.hipGraphGetNodes(graph, nodes, C.byref(n)))
    _LIB.hipKernelNameRefByPtr.restype = C.c_char_p
    names = []
    for node in nodes:
        kind, params = C.c_int(), _KernelNode()
        _ok(_LIB.hipGraphNodeGetType(C.c_void_p(node), C.byref(kind)))
        assert kind.value == 0, "a node that is no kernel"
        _ok(_LIB.hipGraphKernelNodeGetParams(C.c_void_p(node), C.byref(params)))
        names.append(_LIB.hipKernelNameRefByPtr(C.c_void_p(params.func), handle).decode())
    _ok(_LIB.hipGraphDestroy(graph))
    return names
