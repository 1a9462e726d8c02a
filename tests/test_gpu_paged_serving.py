"""The paged operators together (examples/paged_serving.py): a request's outputs do not depend on how its tokens
were cut into steps or on what other requests did, a recorded decode step follows its lengths, and the whole layer
agrees with its steps computed by the oracle from the bits before them."""
import numpy as np
import pytest
import torch

import oracle
import paper_2607_02501_gb300 as emb
from examples.paged_serving import BASE, EPS, PagedLayer
from tests.gpu_util import launches
from tests.paged_util import check, host

pytestmark = pytest.mark.gpu


def _inputs(lens, width, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(n, width, generator=g, device="cuda") for n in lens]


@pytest.mark.parametrize("kw", [dict(), dict(width=512, heads=4, kv_heads=2, head_dim=64, page=32),
                                dict(width=512, heads=4, kv_heads=1, head_dim=256, page=64)])
def test_cutting_into_steps_changes_nothing(cuda_device, kw):
    """Prompts at once, then the same tokens in chunks of any size with idle requests between: the results agree within
    what the differing order of sums and roundings of the steps' kernels allow."""
    lens = [150, 37, 90]
    whole = PagedLayer(requests=3, max_tokens=256, **kw)
    xs = _inputs(lens, whole.width)
    ref = whole.run(torch.cat(xs), lens).split(lens)
    cut = PagedLayer(requests=3, max_tokens=256, **kw)
    at, got = [0, 0, 0], [[], [], []]
    for added in ([100, 0, 1], [1, 1, 1], [0, 30, 60], [40, 1, 0], [9, 5, 28]):
        x = torch.cat([xs[r][at[r]:at[r] + n] for r, n in enumerate(added)])
        out = cut.run(x, added).split(added)
        for r in range(3):
            got[r].append(out[r])
            at[r] += added[r]
    assert at == lens and cut.cached.tolist() == lens
    assert int(cut.used[0]) == sum(-(-n // cut.page) for n in lens) == int(whole.used[0])
    for r in range(3):
        # the layer adds o(attention) to x: attention outputs are bf16 (2^-8), |o| a few units
        err = (torch.cat(got[r]) - ref[r]).abs().max().item()
        assert err < 0.05, f"request {r}: {err}"
        assert (torch.cat(got[r]) - xs[r]).abs().max().item() > 0.1  # (and the layer did something)
    assert emb.emb_paged_status() == emb.EMB_OK and emb.emb_device_status() == emb.EMB_OK


def test_recorded_decode_equals_the_steps_called(cuda_device):
    lens = [40, 3, 130, 17]
    a, b = (PagedLayer(requests=4, max_tokens=256) for _ in range(2))
    xs = torch.cat(_inputs(lens, a.width))
    a.run(xs, lens)
    b.run(xs, lens)
    stream = torch.cuda.Stream()
    buf, rec = b.record_decode(stream)
    for step in range(5):
        x = torch.cat(_inputs([4], a.width, seed=100 + step))
        want = a.run(x, [1, 1, 1, 1])
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            buf["x"].copy_(x)
            rec.launch(stream)
            b.advance(buf)
        torch.cuda.synchronize()
        assert torch.equal(buf["x"], want), step
    assert torch.equal(a.cached, b.cached) and torch.equal(a.table, b.table)
    rec.close()


def test_every_step_against_the_oracle(cuda_device):
    """A mixed step (a chunk, decoded tokens, an idle request) after a prompt, each operator checked from the bits that
    it was given."""
    L = PagedLayer(width=512, heads=8, kv_heads=2, head_dim=128, requests=4, max_tokens=256)
    lens = [100, 20, 64, 5]
    L.run(torch.cat(_inputs(lens, L.width)), lens)
    added = [30, 1, 0, 1]
    b = L.buffers(sum(added))
    b["x"].copy_(torch.cat(_inputs(added, L.width, seed=3)))
    b["added"].copy_(torch.tensor(added, dtype=torch.int32))
    table, used, k0, v0 = L.table.cpu().numpy(), int(L.used[0]), host(L.k_cache), host(L.v_cache)
    L.step(b, 30, window=77)
    torch.cuda.synchronize()
    want = oracle.paged_slots_reference(lens, added, L.free_pages.cpu().numpy(), used, L.page, table, sum(added))
    for got, ref in zip((L.table, b["q_start"], b["kv_len"], b["slots"], b["positions"]), want):
        assert np.array_equal(got.cpu().numpy(), ref)
    assert int(L.used[1]) == want[5]
    pos, slots = want[4][None], want[3]
    axis = np.zeros(64, dtype=int)
    check(host(b["qr"]), *oracle.qk_norm_rope_reference(host(b["q"]), 8, 128, L.q_gamma.cpu().numpy(), EPS, pos, axis, 128, BASE), "q")
    ref, bound = oracle.qk_norm_rope_reference(host(b["k"]), 2, 128, L.k_gamma.cpu().numpy(), EPS, pos, axis, 128, BASE)
    kc, vc = host(L.k_cache), host(L.v_cache)
    check(kc.reshape(-1, 256)[slots], ref, bound, "k")
    v0.reshape(-1, 256)[slots] = host(b["v"])
    assert np.array_equal(vc, v0)
    rest = np.ones(len(k0.reshape(-1, 256)), dtype=bool)
    rest[slots] = False
    assert np.array_equal(kc.reshape(-1, 256)[rest], k0.reshape(-1, 256)[rest])
    check(host(b["a"]), *oracle.paged_attention_reference(host(b["qr"]), kc, vc, want[0], want[1], want[2], 8, 128 ** -0.5, None, 0.0,
                                                          77, 2.0 ** -8), "attention")


@pytest.mark.parametrize("heads,kv_heads,tokens,requests,kernel,clusters", [
    (8, 1, 2, 1, "paged_few_kernel", 1), (16, 1, 1, 1, "paged_few_kernel", 1),          # up to 16 rows of a request
    (8, 1, 50, 1, "paged_few_kernel", 1), (14, 2, 7, 1, "paged_few_kernel", 1),         # more, where all blocks have a cluster
    (8, 8, 1, 400, "paged_few_kernel", 0),                                              # one token of many requests: stretches
    (17, 1, 1, 1, "paged_many_kernel", 0), (8, 1, 3000, 1, "paged_many_kernel", 0)])
def test_which_kernel_a_call_takes(cuda_device, heads, kv_heads, tokens, requests, kernel, clusters):
    T = tokens * requests
    q = torch.zeros(T, heads * 64, dtype=torch.bfloat16, device="cuda")
    cache = torch.zeros(4, 16, kv_heads, 64, dtype=torch.bfloat16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    table, start, kv = torch.zeros(requests, 60, **i32), torch.arange(requests + 1, **i32) * tokens, torch.full((requests,), 900, **i32)
    args = (q, cache, cache, table, start, kv, torch.empty_like(q), 0.1, tokens, emb.paged_workspace())
    got = launches(lambda: emb.emb_paged_attention(*args))
    assert [g[0] for g in got] == [kernel]
    if kernel == "paged_few_kernel":
        assert got[0][1][-1] == clusters  # the last template argument
