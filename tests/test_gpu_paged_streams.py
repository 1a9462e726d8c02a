"""Attention calls whose CTAs join shared items, on several streams at once: each is launched cooperatively, so that all
its CTAs run at once whatever the other streams do."""
import ctypes

import pytest
import torch

import paper_2607_02501_gb300 as emb
from tests.paged_util import Paged, dev_bf16, dev_i32

pytestmark = pytest.mark.gpu
COOPERATIVE = 2  # CU_LAUNCH_ATTRIBUTE_COOPERATIVE

SHAPES = [  # new, kv, H, Hk, d: few rows by stretches, many rows
    ([1], [30000], 8, 1, 128), ([1] * 3, [9000, 30, 16000], 4, 2, 64), ([3], [12000], 4, 1, 256),
    ([700], [3000], 8, 1, 128), ([200, 150], [900, 2000], 7, 1, 64), ([300], [2500], 8, 1, 256)]


def _call(s, ws, stream=None):
    """(arguments on the device, the call)"""
    q = dev_bf16(s.q)
    O = torch.empty_like(q)
    args = (q, dev_bf16(s.k), dev_bf16(s.v), dev_i32(s.table), dev_i32(s.q_start), dev_i32(s.kv), O, s.scale, max(s.new), ws)
    return O, lambda stream=None: emb.emb_paged_attention(*args, stream=stream)


@pytest.mark.parametrize("new,kv,H,Hk,d", SHAPES)
@pytest.mark.parametrize("cap", [0.0, 50.0, 500.0])
def test_launches_that_may_join_are_cooperative(cuda_device, new, kv, H, Hk, d, cap):
    T, R, width = sum(new), len(new), -(-max(kv) // 64)
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.zeros(T, H * d, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(2, 64, Hk, d, dtype=torch.bfloat16, device="cuda")
    args = (q, cache, cache, torch.zeros(R, width, **i32), torch.zeros(R + 1, **i32), torch.zeros(R, **i32), torch.empty_like(q), 0.1, max(new),
            emb.paged_workspace())
    emb.emb_paged_attention(*args, cap=cap)
    cu, stream, graph, count = ctypes.CDLL("libcuda.so.1"), torch.cuda.Stream(), ctypes.c_void_p(), ctypes.c_size_t(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        handle = ctypes.c_void_p(stream.cuda_stream)
        assert cu.cuStreamBeginCapture_v2(handle, 1) == 0
        try:
            emb.emb_paged_attention(*args, cap=cap)
        finally:
            assert cu.cuStreamEndCapture(handle, ctypes.byref(graph)) == 0
    try:
        assert cu.cuGraphGetNodes(graph, None, ctypes.byref(count)) == 0 and count.value == 1
        node, value = ctypes.c_void_p(), (ctypes.c_int * 16)()
        assert cu.cuGraphGetNodes(graph, ctypes.byref(node), ctypes.byref(count)) == 0
        assert cu.cuGraphKernelNodeGetAttribute(node, COOPERATIVE, ctypes.byref(value)) == 0
        assert value[0] == 1
    finally:
        assert cu.cuGraphDestroy(graph) == 0


def test_calls_on_streams_of_different_priority(cuda_device):
    """Every shape on a stream and a workspace of its own, all in flight together, next to a stream of matrix products."""
    low, high = torch.cuda.Stream.priority_range()
    calls = []
    for n, (new, kv, H, Hk, d) in enumerate(SHAPES):
        O, call = _call(Paged(new, kv, H, Hk, d, 64, seed=n), emb.paged_workspace())
        call()
        torch.cuda.synchronize()
        calls.append((O, O.clone(), call, torch.cuda.Stream(priority=high if n % 2 else low)))
        O.fill_(float("nan"))
    other, a = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda").to(torch.bfloat16)
    torch.cuda.synchronize()
    for i in range(40):
        if i % 4 == 0:
            with torch.cuda.stream(other):
                a @ a
        for k in range(len(calls)):
            _, _, call, stream = calls[(k + i) % len(calls)]
            call(stream)
    torch.cuda.synchronize()
    assert emb.emb_paged_status() == emb.EMB_OK
    for O, want, _, _ in calls:
        assert torch.equal(O, want)
