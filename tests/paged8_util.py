"""Inputs of the 8-bit cache's tests: those of the bf16 cache's, encoded block by block."""
import numpy as np
import torch

import oracle
import paper_2607_02501_gb300 as emb
from tests.paged_util import Paged, dev_bf16, dev_i32

# a weight of the value product is rounded once to f16 (half a step)
F16_WEIGHT = 2.0 ** -11


def dev_u8(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, dtype=np.uint8))).cuda()


class Paged8(Paged):
    """A Paged whose cache is encoded when it is first run; k and v are then the codes' values. `spread`: blocks differ by powers of
    two of up to that many."""

    def __init__(self, *args, spread=0, **kw):
        super().__init__(*args, **kw)
        if spread:
            n, page, Hk, _ = self.k.shape
            for x in (self.k, self.v):
                e = self.rng.integers(-spread, spread + 1, (n, page // oracle.paged8.BLOCK, Hk))
                x *= 2.0 ** np.repeat(e, oracle.paged8.BLOCK, axis=1)[..., None]
        self.codes = None

    def encode(self):
        if self.codes is None:
            (kc, ke), (vc, ve) = oracle.paged8_encode(self.k), oracle.paged8_encode(self.v)
            self.codes = [kc, vc, ke, ve]
            self.settle()
        return self.codes

    def settle(self):
        """k and v are what the codes stand for."""
        self.k, self.v = oracle.paged8_values(*self.codes[0::2]), oracle.paged8_values(*self.codes[1::2])

    def garble_unused(self):
        """NaN codes in every place that holds no request's token, any byte as exponent of blocks without one."""
        self.encode()
        used = np.zeros(self.k.shape[:2], dtype=bool)
        for r, n in enumerate(self.kv):
            for pos in range(n):
                used[self.at(r, pos)] = True
        blocks = used.reshape(used.shape[0], -1, oracle.paged8.BLOCK).any(axis=2)
        for c in self.codes[:2]:
            c[~used] = self.rng.choice([0x7F, 0xFF], c[~used].shape)
        for e in self.codes[2:]:
            e[~blocks] = self.rng.integers(0, 256, e[~blocks].shape)
        self.settle()

    spoil_unused = garble_unused

    def run(self, prefix=None, cap=0.0, window=0, max_q=None, pad=0, workspace=None, stream=None):
        self.encode()
        if self.many:
            pad, max_q = 6000, 6000
        q = np.concatenate([self.q[:self.T], np.zeros((pad, self.H * self.d), dtype=np.float32)])
        O = torch.full((q.shape[0], self.H * self.d), float("nan"), dtype=torch.bfloat16, device="cuda")
        ws = emb.paged_workspace() if workspace is None else workspace
        keep = [dev_bf16(q), *map(dev_u8, self.codes), dev_i32(self.table), dev_i32(self.q_start), dev_i32(self.kv)]
        emb.emb_paged8_attention(*keep, O, self.scale, max(self.new) or 1 if max_q is None else max_q, ws,
                                 prefix=None if prefix is None else dev_i32(prefix), cap=cap, window=window, stream=stream)
        torch.cuda.synchronize()
        assert emb.emb_paged_status() == emb.EMB_OK
        assert int(ws[:4096].view(torch.int32).abs().sum()) == 0, "the workspace's flags are handed back at zero"
        return O if not self.many else O[:max(self.T, 1)]
