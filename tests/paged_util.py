"""Inputs of the paged-cache tests: random caches with the pages of several requests in random
order, and the call under test with its outputs poisoned beforehand."""
import numpy as np
import torch

import paper_2607_02501_gb300 as emb


def bf16(a):
    """Values rounded to bf16, as floats."""
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(torch.bfloat16).float().numpy()


def dev_bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).cuda()


def dev_i32(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.int32))).cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


class Paged:
    """A cache of random bf16 values, requests with kv[r] tokens whose last new[r] are the queries. `many`: calls are
    padded to thousands of tokens and hint at as many queries, which small requests take to the kernel for many rows."""

    many = False

    def __init__(self, new, kv, H, Hk, d, page, seed, width=None, spare=3, gain=1.0):
        rng = np.random.default_rng(seed)
        self.rng, self.new, self.kv, self.H, self.Hk, self.d, self.page = rng, list(new), list(kv), H, Hk, d, page
        need = [-(-n // page) for n in kv]
        n_pages = sum(need) + spare
        perm = rng.permutation(n_pages)
        self.table = np.full((len(kv), max(1, max(need)) if width is None else width), -1)
        at = 0
        for r, n in enumerate(need):
            self.table[r, :n] = perm[at:at + n]
            at += n
        self.q_start = np.concatenate([[0], np.cumsum(new)])
        self.T = int(self.q_start[-1])
        self.k = bf16(rng.standard_normal((n_pages, page, Hk, d)) * gain)
        self.v = bf16(rng.standard_normal((n_pages, page, Hk, d)))
        self.q = bf16(rng.standard_normal((max(self.T, 1), H * d)))
        self.scale = d ** -0.5

    def at(self, r, pos):
        """(page, place) of a request's token."""
        return self.table[r, pos // self.page], pos % self.page

    def spoil_unused(self):
        """NaN in every place of the cache that holds no request's token."""
        used = np.zeros(self.k.shape[:2], dtype=bool)
        for r, n in enumerate(self.kv):
            for pos in range(n):
                used[self.at(r, pos)] = True
        self.k[~used] = np.nan
        self.v[~used] = np.nan

    def run(self, prefix=None, cap=0.0, window=0, max_q=None, pad=0, workspace=None, stream=None):
        if self.many:
            pad, max_q = 6000, 6000
        q = np.concatenate([self.q[:self.T], np.zeros((pad, self.H * self.d), dtype=np.float32)])
        O = torch.full((q.shape[0], self.H * self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        ws = emb.paged_workspace() if workspace is None else workspace
        keep = [dev_bf16(q), dev_bf16(self.k), dev_bf16(self.v), dev_i32(self.table), dev_i32(self.q_start),
                dev_i32(self.kv)]
        emb.emb_paged_attention(*keep, O, self.scale, max(self.new) or 1 if max_q is None else max_q, ws,
                                prefix=None if prefix is None else dev_i32(prefix), cap=cap, window=window, stream=stream)
        torch.cuda.synchronize()
        assert emb.emb_paged_status() == emb.EMB_OK
        assert int(ws[:4096].view(torch.int32).abs().sum()) == 0, "the workspace's flags are handed back at zero"
        return O if not self.many else O[:max(self.T, 1)]

    def check(self, weight_error, prefix=None, cap=0.0, window=0, what="", **kw):
        import oracle
        O = self.run(prefix=prefix, cap=cap, window=window, **kw)
        ref, bound = oracle.paged_attention_reference(self.q[:self.T], self.k, self.v, self.table, self.q_start, self.kv,
                                                      self.H, self.scale, prefix, cap, window, weight_error)
        out = host(O)
        check(out[:self.T], ref, bound, what)
        assert (out[self.T:] == 0).all(), "padding rows are zeros"
        return O


def check(out, ref, bound, what):
    assert np.isfinite(out).all(), f"{what}: {int((~np.isfinite(out)).sum())} non-finite outputs"
    bad = np.abs(out - ref) > bound
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} outside, first {np.argwhere(bad)[:4].tolist()} "
                           f"err={np.abs(out - ref)[bad][:4]} bound={bound[bad][:4]}")
