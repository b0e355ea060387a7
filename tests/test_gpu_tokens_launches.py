"""What the token operators launch: the kernels of a call, read from a captured
graph's nodes."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2007_13005_amd import smol, tokens

pytestmark = pytest.mark.gpu


class Dim3(ctypes.Structure):
    _fields_ = [("x", ctypes.c_uint32), ("y", ctypes.c_uint32), ("z", ctypes.c_uint32)]


class KernelNode(ctypes.Structure):  # hipKernelNodeParams
    _fields_ = [("block", Dim3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p),
                ("grid", Dim3), ("params", ctypes.c_void_p), ("shared", ctypes.c_uint32)]


def launches(function):
    """(workgroups, threads of one) of every kernel that function() enqueues."""
    function()  # what a first call makes is not captured
    torch.cuda.synchronize()
    hip = smol.hip_runtime()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        function()
    handle = ctypes.c_void_p(graph.raw_cuda_graph())
    count = ctypes.c_size_t()
    assert hip.hipGraphGetNodes(handle, None, ctypes.byref(count)) == 0
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(handle, nodes, ctypes.byref(count)) == 0
    found = []
    for node in nodes:
        p = KernelNode()
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0
        found.append((p.grid.x * p.grid.y * p.grid.z, p.block.x * p.block.y * p.block.z))
    return found


@pytest.mark.parametrize("n, vocab, dim", [(4, 6400, 4096), (64, 5003, 4096), (777, 5003, 321),
                                           (8, 3000, 2050), (1, 70, 8)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_few_ids_gradient_launches_no_idle_workgroups(n, vocab, dim, accumulate):
    """One launch: workgroups of eight rows and 256 fp32 columns, and the zeros'
    workgroups, 64 KiB each, once."""
    ids = torch.arange(n, device="cuda") % vocab
    dy, out = torch.randn((n, dim), device="cuda"), torch.zeros((vocab, dim), device="cuda")
    room = torch.empty(tokens.embed_workspace_bytes(n, vocab, dim), dtype=torch.uint8,
                       device="cuda")
    found = launches(lambda: tokens.embed_backward(dy, ids, out, accumulate=accumulate,
                                                   workspace=room))
    sums = -(-n // 8) * -(-dim // 256)
    zeros = 0 if accumulate else -(-vocab // max(65536 // (4 * dim), 1))
    assert found == [(sums + zeros, 512)]
