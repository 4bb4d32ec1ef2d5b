"""Plain definitions, in 64 bits, of the calls around a verify step: head norms with the
rotation, changed logits, token counts.  Test infrastructure; shares nothing with the
HIP path."""
from __future__ import annotations

import numpy as np

from .bounded import rotary


def head_norm(x, weight, eps):
    """x [T][H][D]: every head divided by its root mean square, times weight [D]."""
    x = np.asarray(x, dtype=np.float64)
    w = np.ones(x.shape[-1]) if weight is None else np.asarray(weight, dtype=np.float64)
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * w


def norm_rotary(x, weight, eps, pos, freq, axes, interleaved, scale):
    return rotary(head_norm(x, weight, eps), pos, freq, axes, interleaved, scale)


def bits(words, vocab):
    """[..., W] words as truth values [..., vocab]."""
    w = np.asarray(words).view(np.uint32)
    return ((w[..., None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(w.shape[:-1] + (-1,))[..., :vocab] != 0


def words(truth):
    truth = np.asarray(truth)
    wide = np.zeros(truth.shape[:-1] + ((truth.shape[-1] + 31) // 32 * 32,), dtype=np.uint32)
    wide[..., :truth.shape[-1]] = truth
    w = (wide.reshape(truth.shape[:-1] + (-1, 32)) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return w.view(np.int32)


def adjust_logits(logits, tokens, q_start, *, counts=None, seen=None, slots=None, repetition=None, frequency=None,
                  presence=None, bias_start=None, bias_tokens=None, bias_values=None, mask=None, mask_rows=None):
    """(x, size, touched) [T][V]: the changed logits; the sum of the sizes of what was
    multiplied and added, each as often as its rounding counts; what had to change."""
    x = np.array(logits, dtype=np.float64)
    T, V = x.shape
    size, touched = np.zeros_like(x), np.zeros(x.shape, dtype=bool)
    B = len(q_start) - 1
    penal = not (repetition is None and frequency is None and presence is None)
    one = lambda a, i, default: default if a is None else float(a[i])
    for i in range(B):
        r, f, p = one(repetition, i, 1.0), one(frequency, i, 0.0), one(presence, i, 0.0)
        c, prompt = np.zeros(V), np.zeros(V, dtype=bool)
        slot = i if slots is None else int(slots[i])
        if penal and 0 <= slot < counts.shape[0]:
            c = np.where(bits(seen[slot, 1], V), np.maximum(counts[slot], 0), 0).astype(np.float64)
            prompt = bits(seen[slot, 0], V)
        b, b_size, named = np.zeros(V), np.zeros(V), np.zeros(V, dtype=bool)
        if bias_start is not None:
            m = len(bias_tokens)
            for e in range(min(max(bias_start[i], 0), m), min(bias_start[i + 1], m)):
                t = int(bias_tokens[e])
                if 0 <= t < V:
                    b[t] += bias_values[e]
                    b_size[t] += abs(b[t])
                    named[t] = True
        for j in range(q_start[i + 1] - q_start[i]):
            row = q_start[i] + j
            if penal and j > 0 and 0 <= tokens[row] < V:
                c[tokens[row]] += 1
            had = prompt | (c > 0)
            with np.errstate(invalid="ignore"):
                y = np.where(had, np.where(x[row] > 0, x[row] / r, x[row] * r), x[row])
                penalty = np.where(c > 0, f * c + p, 0.0)
                size[row] = np.abs(y) * had + 2 * np.abs(f * c) * (c > 0) + 2 * abs(p) * (c > 0) + b_size + np.abs(b - penalty)
                x[row] = y + (b - penalty)
            touched[row] = (penal & had) | named
            if mask_rows is not None and 0 <= mask_rows[row] < mask.shape[0]:
                out = ~bits(mask[mask_rows[row]], V)
                x[row][out] = -np.inf
                touched[row] |= out
    return x, size, touched


def count_tokens(counts, seen, tokens, start, num=None, slots=None, prompt=False):
    """Copies of counts and seen with the requests' tokens entered."""
    counts, V = np.array(counts), counts.shape[1]
    had = [bits(seen[:, k], V) for k in range(2)]
    for i in range(len(start) - 1):
        slot = i if slots is None else int(slots[i])
        if not 0 <= slot < counts.shape[0]:
            continue
        n = start[i + 1] - start[i]
        for t in tokens[start[i]:start[i] + (n if num is None else min(n, num[i]))]:
            if 0 <= t < V:
                had[0 if prompt else 1][slot, t] = True
                counts[slot, t] += 0 if prompt else 1
    return counts, np.stack([words(h) for h in had], axis=1)
