"""Batches whose groups of requests begin with the same cached tokens."""
from __future__ import annotations

import numpy as np
import torch

import oracle
import paper_2608_24004_amd as av
import workload
from bounded_common import BLOCK, q_start_of


class SharedBatch:
    """groups: [(requests, prefix length)]; S, n: cached keys (with the prefix) and new
    tokens of each request.  Requests in front of and behind the groups: `lead` and the
    rest.  Slots behind a request's keys and spare blocks hold NaN.  wide: block tables
    and bounds of longer requests, so that none counts as short."""

    def __init__(self, seed, groups, S, n, *, hq, hkv, d, dtype, lead=0, sinks=False, spike=False, unmapped=(), wide=False):
        rng = np.random.default_rng(seed)
        self.S, self.n = np.asarray(S, dtype=np.int32), np.asarray(n, dtype=np.int32)
        self.hq, self.hkv, self.d, self.dtype = hq, hkv, d, dtype
        tdt, x = workload.torch_dtype(dtype), workload.elems_per_16b(dtype)
        self.group_start = lead + np.concatenate([[0], np.cumsum([g for g, _ in groups])]).astype(np.int32)
        self.prefix = np.asarray([p for _, p in groups], dtype=np.int32)
        self.q_start = q_start_of(n)
        blocks = -(-self.S // BLOCK)
        own = []
        for i in range(len(S)):
            k = int(np.searchsorted(self.group_start, i, side="right")) - 1
            common = int(self.prefix[k]) // BLOCK if 0 <= k < len(groups) else 0
            own.append((k, common, blocks[i] - common))
        total = sum(max(0, o) for _, _, o in own) + sum(int(p) // BLOCK for p in self.prefix) + 3
        ids = iter(rng.permutation(total).tolist())
        shared = [[next(ids) for _ in range(int(p) // BLOCK)] for p in self.prefix]
        self.table = np.full((len(S), max(1, int(blocks.max(initial=1)))), -1, dtype=np.int32)
        for i, (k, common, o) in enumerate(own):
            row = (shared[k] if common else [])[:blocks[i]] + [next(ids) for _ in range(o)]
            self.table[i, :len(row)] = row
        self.nb = total
        k_cache = torch.full((total, hkv, d // x, BLOCK, x), float("nan"))
        v_cache = torch.full((total, hkv, d, BLOCK), float("nan"))
        for i in range(len(S)):  # whole blocks, then NaN behind the last key
            for b in range(blocks[i]):
                t = min(BLOCK, int(self.S[i]) - b * BLOCK)
                at = self.table[i, b]
                k_cache[at, :, :, :t] = torch.as_tensor(rng.standard_normal((hkv, d // x, t, x)), dtype=torch.float32)
                v_cache[at, :, :, :t] = torch.as_tensor(rng.standard_normal((hkv, d, t)), dtype=torch.float32)
        q = torch.as_tensor(rng.standard_normal((int(self.q_start[-1]), hq, d)), dtype=torch.float32)
        if spike:  # weights that differ by powers of ten
            q *= 4
        self.q, self.k, self.v = q.to(tdt), k_cache.to(tdt), v_cache.to(tdt)
        for i, b in unmapped:
            self.table[i, b] = [-1, total, 2 ** 31 - 1][b % 3]
        if wide:
            self.table = np.pad(self.table, ((0, 0), (0, max(0, 260 - self.table.shape[1]))), constant_values=-1)
        self.max_seq_len = 16 * self.table.shape[1] if wide else int(self.S.max(initial=0))
        self.sinks = torch.as_tensor(rng.standard_normal(hq), dtype=torch.float32) if sinks else None

    @property
    def bounds(self):
        return dict(max_q_len=int(self.n.max(initial=0)), max_seq_len=self.max_seq_len,
                    max_prefix_len=int(self.prefix.max(initial=0)))

    def to(self, device):
        """The call's tensors."""
        arrays = (self.q, self.k, self.v, self.table, self.S, self.q_start, self.group_start, self.prefix)
        return [torch.as_tensor(t).to(device) for t in arrays]

    def call(self, device, args=None, **kw):
        args = self.to(device) if args is None else args
        sinks = None if self.sinks is None else self.sinks.to(device)
        return av.verify_attention_shared(*args, sinks=sinks, **{**self.bounds, **kw})

    def reference(self, scale=0.0):
        """The oracle's output, and the mean size of the values under the same weights."""
        sinks = None if self.sinks is None else self.sinks.double().numpy()
        out = []
        # the definition reads no slot that is not a key: zeros there change nothing
        k, v = torch.nan_to_num(self.k, nan=0.0), torch.nan_to_num(self.v, nan=0.0)
        for values in (v, v.abs()):
            out.append(oracle.attention(
                num_q_heads=self.hq, num_kv_heads=self.hkv, head_dim=self.d, sliding_window=0, scale=scale,
                dtype=workload.dtype_code(self.dtype), q=workload.host_storage(self.q), k_cache=workload.host_storage(k),
                v_cache=workload.host_storage(values), block_tables=self.table, seq_lens=self.S, q_start=self.q_start,
                sinks=sinks))
        return out

    def tolerance(self, ref, size, scale=0.0):
        """A weight's relative error: the score's, a sum of D products in fp32, and three
        roundings of the exponent's size (the factor, the difference, the rescaled
        maximum), and the exponential's own two; in bf16 the weight is rounded to half a
        step before its product.  It counts in the sum of the products and in that of the
        weights, which are sums of S terms in fp32 themselves.  Then the store's half
        step."""
        scale = scale or self.d ** -0.5
        k = torch.nan_to_num(self.k.double(), nan=0.0)
        x = k.shape[-1]
        k_norm = k.permute(0, 1, 3, 2, 4).reshape(-1, k.shape[2] * x).norm(dim=1).max().item()
        q_norm = self.q.double().norm(dim=-1).max().item()
        weight = 2.0 ** -24 * ((self.d + 3) * scale * k_norm * q_norm + 4)
        sums = 2.0 ** -24 * (int(self.S.max()) + 16)
        rounded, store = ((2.0 ** -8, 2.0 ** -8) if self.dtype == "bf16" else (0.0, 2.0 ** -24))
        return (store * np.abs(ref) + size * (rounded + 2 * weight + 2 * sums)) * (1 + 2.0 ** -6)

    def check(self, got, what=""):
        ref, size = self.reference()
        g = got.to(torch.float64).cpu().numpy()
        tol = self.tolerance(ref, size)
        bad = ~(np.abs(g - ref) <= tol)
        assert not bad.any(), "%s %d of %d off, first %s, worst %.3g of its tolerance" % (
            what, bad.sum(), bad.size, np.argwhere(bad)[0], np.nanmax(np.abs(g - ref) / np.maximum(tol, 1e-300)))
