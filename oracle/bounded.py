"""Oracle of the rotary and bounded-cache calls: plain numpy in double precision.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  Caches are given as the
arrays a call takes: k_cache [num_blocks, Hkv, D/x, 16, x], v_cache [num_blocks, Hkv,
D, 16], key_weights and key_order [num_blocks, Hkv, 16]; every function works on
copies and visits one key, row or pair at a time by its definition.

  rotary(...)       a pair (a, b) turned by position * inv_freq
  key_weights(...)  the keys' weights in the counted rows' softmaxes, summed
  evict_plan(...)   the keys to keep, and the slots they are to take
  kv_compact(...)   the moves of such a plan
"""
from __future__ import annotations

import numpy as np

BLOCK = 16


def rotary(x, positions, inv_freq, axes, interleaved, scale=1.0):
    """x [T, H, D] with its first 2 len(axes) dims turned; angles in extended
    precision."""
    y = np.array(x, dtype=np.float64)
    F = len(axes)
    for f in range(F):
        a, b = (2 * f, 2 * f + 1) if interleaved else (f, f + F)
        angle = np.longdouble(positions[axes[f]]) * np.longdouble(inv_freq[f])
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        u, v = y[:, :, a].copy(), y[:, :, b].copy()
        y[:, :, a] = scale * (u * c - v * s)
        y[:, :, b] = scale * (u * s + v * c)
    return y


def _mapped(block, num_blocks):
    return 0 <= block < num_blocks


def key_weights(q, k_cache, weights, order, block_tables, seq_lens, q_start, *, num_rows=None, num_tokens=None,
                sinks=None, scale=0.0, decay=1.0):
    """(new key_weights, new key_order, tolerance): the tolerance bounds what an fp32
    evaluation of the same sums may be off at each key.

    A weight 2^(s - m) / l carries the rounding of its score and of its row's sum.  A
    score is a sum of D products (exact in fp32 for bf16 operands, rounded otherwise):
    at most (D + 2) half steps of 2^-24 relative to the sum of the products' sizes,
    then the scale, the log2(e) and the difference from m, a few half steps of the
    score's size each.  The row's sum adds the same again and one half step per key;
    exponentials, the sum's inverse and the products with it add a few; the sum over
    the rows one per row; the accumulation two of the result."""
    q, k_cache = np.asarray(q, np.float64), np.asarray(k_cache, np.float64)
    w_out, o_out = np.array(weights, np.float64), np.array(order)
    tol = np.zeros_like(w_out)
    T, Hq, D = q.shape
    nb, hkv = k_cache.shape[:2]
    G = Hq // hkv
    scale = scale if scale > 0 else 1.0 / np.sqrt(D)
    half = 2.0 ** -24
    for i in range(len(seq_lens)):
        S, q0 = int(seq_lens[i]), int(q_start[i])
        n = int(q_start[i + 1]) - q0
        count = n if num_rows is None else min(max(int(num_rows[i]), 0), n)
        ids = np.array([block_tables[i][t // BLOCK] for t in range(S)], dtype=np.int64)
        ok = (ids >= 0) & (ids < nb)
        ids, slot = np.where(ok, ids, 0), np.arange(S) % BLOCK
        N = S if num_tokens is None else int(num_tokens[i])
        for g in range(hkv):
            # [S, D]: dim d of slot t at [d / x, t, d % x]
            keys = k_cache[ids, g, :, slot, :].reshape(S, D)
            w, e = np.zeros(S), np.zeros(S)
            for j in range(count):
                p = S - n + j
                see = ok & (np.arange(S) <= p)
                if not see.any():
                    continue
                for h in range(g * G, (g + 1) * G):
                    s = scale * (keys[see] @ q[q0 + j, h])
                    size = scale * (np.abs(keys[see]) @ np.abs(q[q0 + j, h]))
                    top = max(s.max(), -np.inf if sinks is None else sinks[h])
                    ex = np.exp(s - top)
                    total = ex.sum() + (0.0 if sinks is None else np.exp(sinks[h] - top))
                    part = ex / total
                    off = half * ((D + 2) * size.max() + 8 * np.abs(s).max() + 40)
                    w[see] += part
                    e[see] += part * (2 * off + half * (S + 20))
            for t in range(S):
                if not ok[t]:
                    continue
                at = (ids[t], g, slot[t])
                if t >= S - n:
                    w_out[at] = w[t]
                    o_out[at] = N - S + t
                else:
                    w_out[at] = w[t] + (decay * w_out[at] if decay != 0 else 0.0)
                tol[at] = e[t] + half * (count * G * w[t] + 3 * abs(w_out[at]) + 1e-30)
    return w_out, o_out, tol


def evict_plan(weights, order, block_tables, seq_lens, num_blocks, *, max_keys, keep_first=0, keep_recent=0,
               num_tokens=None):
    """(source [B, Hkv, max_keys], new_lens [B])"""
    B, hkv = len(seq_lens), weights.shape[1]
    source = np.full((B, hkv, max_keys), -1, dtype=np.int32)
    new_lens = np.zeros(B, dtype=np.int32)
    for i in range(B):
        S = int(seq_lens[i])
        c = min(S, max_keys)
        N = S if num_tokens is None else int(num_tokens[i])
        new_lens[i] = c
        for g in range(hkv):
            rank = []
            for t in range(S):
                b = int(block_tables[i][t // BLOCK])
                if not _mapped(b, num_blocks):
                    first = (0, 0.0) if t < c else (3, 0.0)
                else:
                    w = float(weights[b, g, t % BLOCK])
                    o = t if order is None else int(order[b, g, t % BLOCK])
                    always = o < keep_first or o >= N - keep_recent
                    first = (0, 0.0) if always else (1, 0.0) if np.isnan(w) else (2, -w)
                rank.append(first + (t,))
            kept = {r[2] for r in sorted(rank)[:c]}
            movers = sorted(t for t in kept if t >= c)
            for d in range(c):
                source[i, g, d] = d if d in kept else movers.pop(0)
            assert not movers
    return source, new_lens


def kv_compact(k_cache, v_cache, weights, order, block_tables, source, new_lens):
    """Copies of the four arrays after the moves of `source`."""
    k, v, w, o = (np.array(x) for x in (k_cache, v_cache, weights, order))
    nb = k.shape[0]
    B, hkv, C = source.shape
    for i in range(B):
        width = len(block_tables[i])
        for g in range(hkv):
            for d in range(min(int(new_lens[i]), C)):
                s = int(source[i, g, d])
                if s == d or s < 0 or s >= BLOCK * width or d >= BLOCK * width:
                    continue
                fb, tb = int(block_tables[i][s // BLOCK]), int(block_tables[i][d // BLOCK])
                if not (_mapped(fb, nb) and _mapped(tb, nb)):
                    continue
                ft, tt = s % BLOCK, d % BLOCK
                k[tb, g, :, tt] = k_cache[fb, g, :, ft]
                v[tb, g, :, tt] = v_cache[fb, g, :, ft]
                w[tb, g, tt] = weights[fb, g, ft]
                o[tb, g, tt] = order[fb, g, ft]
    return k, v, w, o
