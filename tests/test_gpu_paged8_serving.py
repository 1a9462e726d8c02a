"""The 8-bit cache's operators together (examples/paged_serving.py with bits=8): steps cut in any way agree, a recorded decode step
equals the calls, a mixed step agrees with the oracle operator by operator, calls on streams of their own and calls that take
turns on one workspace do not meet, and which kernel a call takes."""
import ctypes
import subprocess
import sys

import numpy as np
import pytest
import torch

import __graft_entry__ as entry
import oracle
import paper_2607_02501_gb300 as emb
from examples.paged_serving import BASE, EPS, PagedLayer
from tests.gpu_util import launches
from tests.paged_util import check, dev_bf16, dev_i32, host
from tests.paged8_util import F16_WEIGHT, Paged8, dev_u8
from tests.test_gpu_paged_serving import _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(width=512, heads=4, kv_heads=2, head_dim=64, page=32),
                                dict(width=512, heads=4, kv_heads=1, head_dim=256, page=64)])
def test_cutting_into_steps(cuda_device, kw):
    """Prompts at once, then the same tokens in chunks of any size with idle requests between. The projections of another number of
    tokens round some keys and values to the neighbouring bf16 number, which moves some codes by a step (2^-3 of the value):
    beside the 0.05 of the bf16 cache's test, 0.1 for those."""
    lens = [150, 37, 90]
    whole, cut = (PagedLayer(requests=3, max_tokens=256, bits=8, **kw) for _ in range(2))
    xs = _inputs(lens, whole.width)
    ref = whole.run(torch.cat(xs), lens).split(lens)
    at, got = [0, 0, 0], [[], [], []]
    for added in ([100, 0, 1], [1, 1, 1], [0, 30, 60], [40, 1, 0], [9, 5, 28]):
        out = cut.run(torch.cat([xs[r][at[r]:at[r] + n] for r, n in enumerate(added)]), added).split(added)
        for r in range(3):
            got[r].append(out[r])
            at[r] += added[r]
    assert at == lens and cut.cached.tolist() == lens
    for r in range(3):
        assert (torch.cat(got[r]) - ref[r]).abs().max().item() < 0.15
        assert (torch.cat(got[r]) - xs[r]).abs().max().item() > 0.1  # (and the layer did something)
    assert emb.emb_paged_status() == emb.EMB_OK and emb.emb_device_status() == emb.EMB_OK


def test_recorded_decode_equals_the_steps_called(cuda_device):
    """Also where a block is begun, gone on with and filled, and while eager steps of another layer run beside the replays."""
    lens = [40, 3, 130, 14]
    a, b, other = (PagedLayer(requests=4, max_tokens=256, bits=8) for _ in range(3))
    xs = torch.cat(_inputs(lens, a.width))
    for layer in (a, b, other):
        layer.run(xs, lens)
    stream = torch.cuda.Stream()
    buf, rec = b.record_decode(stream)
    for step in range(6):
        x = torch.cat(_inputs([4], a.width, seed=100 + step))
        want = a.run(x, [1, 1, 1, 1])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            buf["x"].copy_(x)
            rec.launch(stream)
            b.advance(buf)
        got = other.run(x, [1, 1, 1, 1])
        torch.cuda.synchronize()
        assert torch.equal(buf["x"], want) and torch.equal(got, want), step
    for u, v in zip(a.cache, b.cache):
        assert torch.equal(u, v)
    assert torch.equal(a.cached, b.cached) and torch.equal(a.table, b.table)
    rec.close()


def test_two_recordings_take_turns(cuda_device):
    """Two recorded steps on one layer's cache and workspace, launched in turn on one stream."""
    a, b = (PagedLayer(requests=2, max_tokens=512, bits=8) for _ in range(2))
    xs = torch.cat(_inputs([100, 300], a.width))
    a.run(xs, [100, 300])
    b.run(xs, [100, 300])
    stream = torch.cuda.Stream()
    recs = [b.record_decode(stream) for _ in range(2)]
    for step in range(5):
        x = torch.cat(_inputs([2], a.width, seed=step))
        want = a.run(x, [1, 1])
        torch.cuda.synchronize()
        buf, rec = recs[step % 2]
        with torch.cuda.stream(stream):
            buf["x"].copy_(x)
            rec.launch(stream)
            b.advance(buf)
        torch.cuda.synchronize()
        assert torch.equal(buf["x"], want), step
    for _, rec in recs:
        rec.close()


def test_every_step_against_the_oracle(cuda_device):
    """A mixed step (a chunk, decoded tokens, an idle request) after a prompt, each operator checked from the bits it was given."""
    L = PagedLayer(width=512, heads=8, kv_heads=2, head_dim=128, requests=4, max_tokens=256, bits=8)
    lens = [100, 20, 64, 5]
    L.run(torch.cat(_inputs(lens, L.width)), lens)
    added = [30, 1, 0, 1]
    b = L.buffers(sum(added))
    b["x"].copy_(torch.cat(_inputs(added, L.width, seed=3)))
    b["added"].copy_(torch.tensor(added, dtype=torch.int32))
    before = [c.cpu().numpy() for c in L.cache]
    table, used = L.table.cpu().numpy(), int(L.used[0])
    L.step(b, 30, window=77)
    torch.cuda.synchronize()
    want = oracle.paged_slots_reference(lens, added, L.free_pages.cpu().numpy(), used, L.page, table, sum(added))
    kc, vc, ke, ve = (c.cpu().numpy() for c in L.cache)
    want_c, want_e = oracle.paged8_store_reference(host(b["v"]).reshape(-1, 2, 128), before[1], before[3], want[3])
    assert np.array_equal(ve, want_e) and np.array_equal(oracle.paged8_values(vc, ve), oracle.paged8_values(want_c, want_e))
    K, V = oracle.paged8_values(kc, ke), oracle.paged8_values(vc, ve)
    axis, turns = [0] * 64, [int(x) % 2 ** 64 for x in L.turns.tolist()]
    y, err = oracle.norm_turn_reference(host(b["q"]), 8, 128, L.q_gamma.cpu().numpy(), EPS, want[4][None], axis, turns)
    check(host(b["qr"]), y.reshape(sum(added), -1), oracle.bf16_bound(y, err).reshape(sum(added), -1), "q")
    bf, _ = oracle.qk_norm_rope_reference(host(b["q"]), 8, 128, L.q_gamma.cpu().numpy(), EPS, want[4][None], np.zeros(64, dtype=int), 128, BASE)
    assert np.abs(bf - y.reshape(bf.shape)).max() < 1e-6  # (the bf16 cache's rotation)
    y, err = oracle.norm_turn_reference(host(b["k"]), 2, 128, L.k_gamma.cpu().numpy(), EPS, want[4][None], axis, turns)
    got = K.reshape(-1, 2, 128)[want[3]]
    unit = 2.0 ** oracle.exponent_of(ke).reshape(-1, 2)[want[3] // 16][..., None]
    assert (np.abs(got - y) <= err + np.maximum(2.0 ** -4 * (np.abs(y) + err), 2.0 ** -10 * unit)).all()
    check(host(b["a"]), *oracle.paged_attention_reference(host(b["qr"]), K, V, want[0], want[1], want[2], 8, 128 ** -0.5, None, 0.0, 77,
                                                          F16_WEIGHT), "attention")


def test_one_workspace_for_both_caches_in_turn(cuda_device):
    from tests.paged_util import Paged
    ws = emb.paged_workspace()
    for new, kv in (([1], [9000]), ([300], [2500])):
        a, b = Paged(new, kv, 8, 1, 128, 64, seed=1), Paged8(new, kv, 8, 1, 128, 64, seed=2)
        want = a.run(workspace=ws), b.run(workspace=ws)
        for _ in range(3):
            assert torch.equal(a.run(workspace=ws), want[0]) and torch.equal(b.run(workspace=ws), want[1])


SHAPES = [  # new, kv, H, Hk, d: few rows by stretches, many rows
    ([1], [30000], 8, 1, 128), ([1] * 3, [9000, 30, 16000], 4, 2, 64), ([3], [12000], 4, 1, 256),
    ([700], [3000], 8, 1, 128), ([200, 150], [900, 2000], 7, 1, 64), ([300], [2500], 8, 1, 256)]


def _args(s, ws):
    q = dev_bf16(s.q)
    return (q, *map(dev_u8, s.encode()), dev_i32(s.table), dev_i32(s.q_start), dev_i32(s.kv), torch.empty_like(q), s.scale, max(s.new), ws)


def test_calls_on_streams_of_different_priority(cuda_device):
    """Every shape on a stream and a workspace of its own, all in flight together, next to a stream of matrix products."""
    low, high = torch.cuda.Stream.priority_range()
    calls = []
    for n, (new, kv, H, Hk, d) in enumerate(SHAPES):
        args = _args(Paged8(new, kv, H, Hk, d, 64, seed=n), emb.paged_workspace())
        emb.emb_paged8_attention(*args)
        torch.cuda.synchronize()
        calls.append((args, args[8].clone(), torch.cuda.Stream(priority=high if n % 2 else low)))
        args[8].fill_(float("nan"))
    other, a = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda").to(torch.bfloat16)
    torch.cuda.synchronize()
    for i in range(40):
        if i % 4 == 0:
            with torch.cuda.stream(other):
                a @ a
        for k in range(len(calls)):
            args, _, stream = calls[(k + i) % len(calls)]
            emb.emb_paged8_attention(*args, stream=stream)
    torch.cuda.synchronize()
    assert emb.emb_paged_status() == emb.EMB_OK
    for args, want, _ in calls:
        assert torch.equal(args[8], want)


@pytest.mark.parametrize("new,kv,H,Hk,d", SHAPES)
@pytest.mark.parametrize("cap", [0.0, 50.0, 500.0])
def test_launches_that_may_join_are_cooperative(cuda_device, new, kv, H, Hk, d, cap):
    args = _args(Paged8(new, kv, H, Hk, d, 64, seed=3), emb.paged_workspace())
    emb.emb_paged8_attention(*args, cap=cap)
    cu, stream, graph, count = ctypes.CDLL("libcuda.so.1"), torch.cuda.Stream(), ctypes.c_void_p(), ctypes.c_size_t(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        handle = ctypes.c_void_p(stream.cuda_stream)
        assert cu.cuStreamBeginCapture_v2(handle, 1) == 0
        try:
            emb.emb_paged8_attention(*args, cap=cap)
        finally:
            assert cu.cuStreamEndCapture(handle, ctypes.byref(graph)) == 0
    try:
        assert cu.cuGraphGetNodes(graph, None, ctypes.byref(count)) == 0 and count.value == 1
        node, value = ctypes.c_void_p(), (ctypes.c_int * 16)()
        assert cu.cuGraphGetNodes(graph, ctypes.byref(node), ctypes.byref(count)) == 0
        assert cu.cuGraphKernelNodeGetAttribute(node, 2, ctypes.byref(value)) == 0  # CU_LAUNCH_ATTRIBUTE_COOPERATIVE
        assert value[0] == 1
    finally:
        assert cu.cuGraphDestroy(graph) == 0


@pytest.mark.parametrize("R,H,Hk,d,new,keys,kernel,clusters", [
    (1, 8, 1, 64, 2, 900, "paged_codes_few_kernel", 1), (1, 8, 1, 64, 50, 900, "paged_codes_few_kernel", 1),   # clusters
    (400, 8, 8, 64, 1, 900, "paged_codes_few_kernel", 0), (32, 16, 2, 128, 4, 8000, "paged_codes_few_kernel", 0),   # stretches; up to 32 rows
    (1, 16, 2, 256, 8, 16000, "paged_codes_few_kernel", 0),                                                # few blocks: up to 64
    (32, 16, 2, 256, 4, 8000, "paged_codes_many_kernel", None), (32, 16, 2, 128, 8, 8000, "paged_codes_many_kernel", None),
    (1, 17, 1, 64, 1, 900, "paged_codes_many_kernel", None), (1, 8, 1, 64, 3000, 900, "paged_codes_many_kernel", None)])
def test_which_kernel_a_call_takes(cuda_device, R, H, Hk, d, new, keys, kernel, clusters):
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.zeros(R * new, H * d, dtype=torch.bfloat16, device="cuda")
    cache = emb.paged8_cache(4, 16, Hk, d)
    args = (q, *cache, torch.zeros(R, -(-keys // 16), **i32), torch.arange(R + 1, **i32) * new, torch.full((R,), keys, **i32), torch.empty_like(q), 0.1, new,
            emb.paged_workspace())
    for cap in (0.0, 50.0, 500.0):
        emb.emb_paged8_attention(*args, cap=cap)
        (name, template, _), = launches(lambda: emb.emb_paged8_attention(*args, cap=cap))
        assert name == kernel
        if clusters is not None:
            assert template[-1] == clusters


def test_timeout_is_reported(cuda_device):
    """A join that gives up, in the workspace that both caches' calls share; after the flags are zeroed all is as before."""
    s = Paged8([1], [9000], 8, 1, 128, 64, seed=4)
    ws = emb.paged_workspace()
    want = s.run(workspace=ws)
    emb.emb_paged_selftest_wait_timeout(ws, 100000)
    assert emb.emb_paged_status() == emb.EMB_ETIMEOUT
    ws[:4096] = 0
    assert torch.equal(s.run(workspace=ws), want)


def test_smoke_step_reaches_every_kernel(cuda_device):
    _, calls = entry.paged8_step()
    for call in calls:  # (functions are set up at their first call, outside of a capture)
        call()
    got = [k[0][0] for k in map(launches, calls)]
    assert got == ["paged_slots_kernel", "paged_codes_store_kernel", "paged_codes_store_kernel", "paged_codes_few_kernel", "paged_codes_many_kernel", "paged_codes_read_kernel"]
    entry.smoke_paged8()


def test_example_runs(cuda_device):
    for bits in ("8", "16"):
        out = subprocess.run([sys.executable, "examples/paged_serving.py", "--steps", "3", "--bits", bits], capture_output=True, text=True, timeout=300)
        assert out.returncode == 0 and "lengths [819, 53, 303, 10]" in out.stdout, out.stderr[-2000:]
