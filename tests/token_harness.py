"""Caches for the tests of the calls that decode one token at a time: the same bytes for the oracle (float64) and
for the library.  Pages are scattered over the pool by a permutation; memory that holds nothing (rows behind
kv_len, pages of nobody) is NaN, so that a value read from there shows."""
from __future__ import annotations

import numpy as np
import torch

from oracle import flowblock_oracle as O
from paper_2607_17652_b200 import binding as B
from paper_2607_17652_b200 import synth
from tests import harness as H

PAGE = 64
NAN_E4M3 = 0x7F


class Case:
    def __init__(self, lens, heads=(8, 2, 128), fp8=False, seed=0, pages_per_req=None, spare_pages=3, fill=True):
        self.hq, self.hkv, self.d = heads
        self.lens = np.asarray(lens, np.int32)
        self.R, self.fp8 = len(lens), fp8
        rng = np.random.default_rng([seed, self.R, self.hq, self.d])
        need = np.maximum(0, -(-self.lens // PAGE))
        self.width = pages_per_req or max(1, int(need.max()))
        self.cap = self.width * PAGE
        self.num_pages = int(self.R * self.width) + spare_pages
        perm = rng.permutation(self.num_pages)[:self.R * self.width]
        self.page_table = perm.reshape(self.R, self.width).astype(np.int32)
        gen = torch.Generator().manual_seed(seed)
        self.gen, self.rng = gen, rng
        shape = (self.num_pages, self.hkv, PAGE, self.d)
        self.scales = None
        if fp8:
            self.scales = [(0.01 + 0.02 * torch.rand(self.hkv, generator=gen)).float() for _ in range(2)]
            # every finite code
            k, v = (torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8) for _ in range(2))
            for x in (k, v):
                x[(x & 0x7F) == 0x7F] = 0x3A
            # (a few large codes would decide every softmax: keep most keys moderate)
            k &= 0xBF
        else:
            k, v = (torch.randn(shape, generator=gen).to(torch.bfloat16) for _ in range(2))
        self.k_pool, self.v_pool = k, v
        if fill:
            self._poison()
        self.k_new, self.v_new = (torch.randn(self.R, self.hkv, self.d, generator=gen).to(torch.bfloat16) for _ in range(2))
        self.q = torch.randn(self.R, self.hq, self.d, generator=gen).to(torch.bfloat16)
        self.tok_pos = (self.lens - 1 + rng.integers(0, 5000, self.R)).astype(np.int32)
        self.kv_pos = rng.integers(0, 40000, (self.R, self.hkv, self.cap)).astype(np.int32)
        self.kv_weight = np.exp(rng.normal(size=(self.R, self.hkv, self.cap)) * 1.5).astype(np.float32)

    def _poison(self):
        held = np.zeros((self.num_pages, PAGE), bool)
        for r in range(self.R):
            for j in range(max(0, int(self.lens[r]))):
                held[self.page_table[r, j // PAGE], j % PAGE] = True
        bad = torch.from_numpy(~held)[:, None, :, None].expand(self.k_pool.shape)
        for x in (self.k_pool, self.v_pool):
            x[bad] = NAN_E4M3 if self.fp8 else float("nan")

    def cfg(self, **over):
        c = dict(max_requests=self.R, wmax=1, block_len=128 * self.hkv // self.hq, n_q_heads=self.hq, n_kv_heads=self.hkv,
                 head_dim=self.d, page_size=PAGE, num_pages=self.num_pages, max_pages_per_req=self.width, vocab=1024,
                 mask_id=1023, eos_id=-1, max_blocks=1, s_pe=0, tau_mask=0.9, tau_edit=0.95, theta_spawn=0.5, sm_scale=0.0)
        c.update(over)
        return c

    def oracle_cfg(self, **over):
        return O.Config(**self.cfg(**over))

    def context(self, tuning=None, **over):
        if self.fp8:
            over = dict(dict(window_in_pages=1, kv_fp8=1), **over)
        return B.Context(tuning=tuning, **self.cfg(**over))

    def pools64(self):
        """What the pages hold, in float64 (8-bit pages: decoded and scaled)."""
        if not self.fp8:
            return H.f64(self.k_pool), H.f64(self.v_pool)
        return tuple(O.e4m3_decode(p.numpy()) * s.double().numpy()[None, :, None, None]
                     for p, s in zip((self.k_pool, self.v_pool), self.scales))

    def device(self, dev="cuda:0", records=True):
        """(CacheState, k_pool, v_pool) on the GPU."""
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)
        cache = B.CacheState(t(self.lens), t(self.tok_pos), t(self.kv_pos) if records else None,
                             t(self.kv_weight) if records else None, t(self.page_table))
        return cache, self.k_pool.to(dev), self.v_pool.to(dev)

    def dev_scales(self, dev="cuda:0"):
        if not hasattr(self, "_dev_scales"):
            self._dev_scales = [s.to(dev) for s in self.scales]
        return self._dev_scales


def bits(t: torch.Tensor) -> np.ndarray:
    t = t.cpu()
    return (t if t.dtype == torch.uint8 else t.view(torch.int16)).numpy()


__all__ = ["Case", "PAGE", "bits", "synth"]
