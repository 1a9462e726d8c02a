"""Several requests served step by step through one transformer layer over a paged key/value cache.

Each step takes the new tokens of every request (a prompt, a chunk, a decoded token, or none) and runs

    emb_paged_slots                      pages, slots and positions of the step, from the lengths
    emb_rmsnorm -> q, k, v (bf16)        the layer's norm and block-quantised projections
    emb_qk_norm_rope                     q and k normed per head and rotated, k and v into the cache
    emb_paged_attention                  every new token over its request's whole history
    o (+ residual)                       the output projection into the residual stream

on one stream, with no host synchronisation in between; the lengths stay on the device, and a step of fixed
size (a decode step) can be recorded once and replayed (`record_decode`).

    python examples/paged_serving.py [--steps 8]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2607_02501_gb300 as emb  # noqa: E402

EPS, BASE = 1e-6, 10000.0


class PagedLayer:
    """One layer (width, heads, key/value heads, head dim) with random Q8_0 weights, and the cache and bookkeeping of
    `requests` requests with up to `max_tokens` tokens each."""

    def __init__(self, width=1024, heads=8, kv_heads=1, head_dim=128, requests=4, max_tokens=2048, page=16, seed=0):
        self.width, self.heads, self.kv_heads, self.head_dim, self.requests, self.page = width, heads, kv_heads, head_dim, requests, page
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        dev = {"device": "cuda"}
        qd, kd = heads * head_dim, kv_heads * head_dim
        self.shapes = {"q": (qd, width), "k": (kd, width), "v": (kd, width), "o": (width, qd)}
        self.weights = {n: emb.quantize(emb.EMB_Q8_0, torch.randn(*s, generator=g, **dev) * s[1] ** -0.5)
                        for n, s in self.shapes.items()}
        self.norm = 1.0 + 0.1 * torch.randn(width, generator=g, **dev)
        self.q_gamma = 1.0 + 0.1 * torch.randn(head_dim, generator=g, **dev)
        self.k_gamma = 1.0 + 0.1 * torch.randn(head_dim, generator=g, **dev)
        pages = -(-max_tokens // page)
        n_pages = requests * pages
        self.k_cache = torch.zeros(n_pages, page, kv_heads, head_dim, dtype=torch.bfloat16, **dev)
        self.v_cache = torch.zeros_like(self.k_cache)
        self.table = torch.full((requests, pages), -1, dtype=torch.int32, **dev)
        # pages are handed out in an order of their own
        self.free_pages = torch.randperm(n_pages, generator=g, **dev).to(torch.int32)
        self.used = torch.zeros(2, dtype=torch.int32, **dev)      # entries taken before and after a step
        self.cached = torch.zeros(requests, dtype=torch.int32, **dev)
        self.workspace = emb.paged_workspace()

    def buffers(self, tokens):
        """A step's buffers for that many tokens."""
        dev, bf = {"device": "cuda"}, torch.bfloat16
        qd, kd = self.heads * self.head_dim, self.kv_heads * self.head_dim
        return {"x": torch.zeros(tokens, self.width, **dev), "h": torch.empty(tokens, self.width, dtype=bf, **dev),
                "q": torch.empty(tokens, qd, dtype=bf, **dev), "k": torch.empty(tokens, kd, dtype=bf, **dev),
                "v": torch.empty(tokens, kd, dtype=bf, **dev), "qr": torch.empty(tokens, qd, dtype=bf, **dev),
                "a": torch.empty(tokens, qd, dtype=bf, **dev),
                "added": torch.zeros(self.requests, dtype=torch.int32, **dev),
                "q_start": torch.empty(self.requests + 1, dtype=torch.int32, **dev),
                "kv_len": torch.empty(self.requests, dtype=torch.int32, **dev),
                "slots": torch.empty(tokens, dtype=torch.int64, **dev),
                "positions": torch.empty(tokens, dtype=torch.int32, **dev)}

    def step(self, b, max_q, prefix=None, cap=0.0, window=0, stream=None):
        """One step on the buffers `b`, whose x (the residual stream, updated in place) and added hold its tokens."""
        T = b["x"].shape[0]
        H, Hk, d, w = self.heads, self.kv_heads, self.head_dim, self.weights
        emb.emb_paged_slots(self.cached, b["added"], self.free_pages, self.used[:1], self.table, b["q_start"], b["kv_len"],
                            b["slots"], b["positions"], self.used[1:], self.page, stream=stream)
        emb.emb_rmsnorm(b["x"], self.norm, b["h"], EPS, stream=stream)
        emb.emb_qlayer_seq([(emb.EMB_Q8_0, w[n], *self.shapes[n], b["h"], b[n], emb.EMB_EPI_BF16) for n in "qkv"], T, stream=stream)
        emb.emb_qk_norm_rope(b["q"], b["k"], b["v"], b["qr"], self.k_cache, self.v_cache, b["slots"], b["positions"],
                             q_gamma=self.q_gamma, k_gamma=self.k_gamma, eps=EPS, base=BASE, stream=stream)
        emb.emb_paged_attention(b["qr"], self.k_cache, self.v_cache, self.table, b["q_start"], b["kv_len"], b["a"], d ** -0.5,
                                max_q, self.workspace, prefix=prefix, cap=cap, window=window, stream=stream)
        emb.emb_qlayer_seq([(emb.EMB_Q8_0, w["o"], *self.shapes["o"], b["a"], b["x"], emb.EMB_EPI_ADD)], T, stream=stream)

    def advance(self, b):
        """Takes the step's tokens and pages over into the next step (on the current stream)."""
        self.cached.copy_(b["kv_len"])
        self.used[:1].copy_(self.used[1:])

    def run(self, x, added, **kw):
        """A step of new size: x fp32 [tokens][width] in request order; returns the residual stream after the layer."""
        b = self.buffers(x.shape[0])
        b["x"].copy_(x)
        b["added"].copy_(torch.tensor(added, dtype=torch.int32))
        self.step(b, max(1, max(added)), **kw)
        self.advance(b)
        return b["x"]

    def record_decode(self, stream, **kw):
        """A decode step (one token per request) recorded on `stream`: fill b["x"], launch, advance."""
        b = self.buffers(self.requests)
        b["added"].fill_(1)
        torch.cuda.synchronize()
        with emb.Recording(stream, keep=[self, b]) as rec:
            self.step(b, 1, stream=stream, **kw)
        return b, rec


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=8)
    steps = ap.parse_args().steps
    layer = PagedLayer(requests=4)
    prompts = [816, 50, 300, 7]
    x = torch.randn(sum(prompts), layer.width, device="cuda")
    layer.run(x, prompts)
    stream = torch.cuda.Stream()
    b, rec = layer.record_decode(stream)
    with torch.cuda.stream(stream):
        start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        start.record()
        for _ in range(steps):
            b["x"].normal_()
            rec.launch(stream)
            layer.advance(b)
        end.record()
    torch.cuda.synchronize()
    assert emb.emb_paged_status() == emb.EMB_OK and emb.emb_device_status() == emb.EMB_OK
    print(f"{layer.requests} requests, {sum(prompts)} prompt tokens, {steps} decode steps: "
          f"{start.elapsed_time(end) / steps * 1e3:.1f} us a step; lengths {layer.cached.tolist()}, pages taken {int(layer.used[0])}")
    rec.close()


if __name__ == "__main__":
    main()
