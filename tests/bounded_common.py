"""Inputs of the rotary and bounded-cache tests."""
from __future__ import annotations

import numpy as np
import torch

import workload

BLOCK = 16


class Cache:
    """A layer's paged cache with key weights and ordinals, every slot behind a
    request's keys (and every spare block) holding NaN, on the CPU; `to` copies it."""

    def __init__(self, rng, S, *, hkv, d, dtype, spare=3, unmapped=0, lost=None):
        self.S = np.asarray(S, dtype=np.int32)
        self.hkv, self.d, self.dtype = hkv, d, workload.torch_dtype(dtype)
        x = workload.elems_per_16b(dtype)
        blocks = -(-self.S // BLOCK)
        self.nb = int(blocks.sum()) + spare
        ids = rng.permutation(self.nb).astype(np.int32)
        self.block_tables = np.full((len(S), max(1, int(blocks.max(initial=0)))), -1, dtype=np.int32)
        self.k = torch.full((self.nb, hkv, d // x, BLOCK, x), float("nan"), dtype=self.dtype)
        self.v = torch.full((self.nb, hkv, d, BLOCK), float("nan"), dtype=self.dtype)
        self.w = torch.full((self.nb, hkv, BLOCK), float("nan"))
        self.o = torch.full((self.nb, hkv, BLOCK), -77, dtype=torch.int32)
        self.tokens = self.S + (0 if lost is None else np.asarray(lost, dtype=np.int32))
        off = 0
        for i, s in enumerate(self.S):
            self.block_tables[i, :blocks[i]] = ids[off:off + blocks[i]]
            off += blocks[i]
            order = np.stack([np.sort(rng.choice(self.tokens[i], size=s, replace=False)) for _ in range(hkv)]) \
                if lost is not None and s else np.tile(np.arange(s), (hkv, 1))
            for t in range(s):
                b, slot = int(self.block_tables[i, t // BLOCK]), t % BLOCK
                self.k[b, :, :, slot] = torch.as_tensor(rng.standard_normal((hkv, d // x, x))).to(self.dtype)
                self.v[b, :, :, slot] = torch.as_tensor(rng.standard_normal((hkv, d))).to(self.dtype)
                self.w[b, :, slot] = torch.as_tensor(rng.exponential(size=hkv), dtype=torch.float32)
                self.o[b, :, slot] = torch.as_tensor(order[:, t].astype(np.int32))
        for _ in range(unmapped):  # ids outside the cache inside a request's keys
            i = int(rng.integers(len(S)))
            if blocks[i]:
                self.block_tables[i, int(rng.integers(blocks[i]))] = int(rng.choice([-1, self.nb, 10 ** 9]))

    def to(self, device):
        return [torch.as_tensor(t).to(device).clone() for t in (self.k, self.v, self.w, self.o, self.block_tables, self.S)]

    def numpy(self):
        return [t.to(torch.float64).numpy() if t.is_floating_point() else t.numpy()
                for t in (self.k, self.v, self.w, self.o)]


def q_start_of(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def bits(t):
    """A tensor's storage bits, on the CPU."""
    t = t.detach().cpu().contiguous()
    return t.view({2: torch.int16, 4: torch.int32}[t.element_size()]).numpy()
