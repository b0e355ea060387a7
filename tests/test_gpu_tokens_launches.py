"""What the token operators launch: the kernels of a call, read from a captured
graph's nodes."""
from __future__ import annotations

import ctypes

import pytest
import torch

from paper_2007_13005_amd import smol, tokens
from tests import tokens_util as ref

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


@pytest.mark.parametrize("n, dim, dtype, alone", [
    (1024, 1024, torch.bfloat16, True), (1024, 2048, torch.bfloat16, True),
    (512, 4096, torch.float32, True), (8, 65536, torch.float32, True),
    (1024, 3, torch.float32, True), (1024, 2048, torch.float32, False),
    (1024, 4096, torch.float32, False), (256, 65536, torch.float32, False),
    (1025, 8, torch.float32, False)])
def test_few_ids_gradient_in_one_launch_where_that_is_faster(n, dim, dtype, alone):
    """Not for many rows of many columns, whose workgroups would each look at
    all ids: those are counted, summed and joined (256 rows of 65536 fp32
    columns, 93 us in one launch, 38 in three)."""
    vocab = 100
    ids = torch.arange(n, device="cuda") % vocab
    dy = torch.randn((n, dim), device="cuda").to(dtype)
    out = torch.zeros((vocab, dim), device="cuda")
    room = torch.empty(tokens.embed_workspace_bytes(n, vocab, dim), dtype=torch.uint8,
                       device="cuda")
    found = launches(lambda: tokens.embed_backward(dy, ids, out, accumulate=True, workspace=room))
    assert len(found) == (1 if alone else 3)
    tokens.embed_backward(dy, ids, out, 0.5, workspace=room)
    want, bound = ref.embed_backward(dy.cpu(), ids.cpu(), vocab, 0.5)
    ref.close(out, want, bound, "embed grad")
