"""The oracle of the rotary and bounded-cache calls against other statements of the
same definitions."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from bounded_common import Cache, q_start_of
from oracle import bounded


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 64))
    pos = rng.integers(-50, 5000, size=(2, 5))
    axes = [f % 2 for f in range(24)]
    freq = 10000.0 ** (-np.arange(24) / 24)
    y = bounded.rotary(x, pos, freq, axes, interleaved, 1.5)
    even, odd = (slice(0, 48, 2), slice(1, 48, 2)) if interleaved else (slice(0, 24), slice(24, 48))
    angle = pos[axes].T * freq
    z = 1.5 * (x[..., even] + 1j * x[..., odd]) * np.exp(1j * angle)[:, None, :]
    np.testing.assert_allclose(y[..., even], z.real, atol=1e-11)
    np.testing.assert_allclose(y[..., odd], z.imag, atol=1e-11)
    np.testing.assert_array_equal(y[..., 48:], x[..., 48:])


def test_key_weights_are_column_sums_of_the_softmax():
    rng = np.random.default_rng(2)
    S, n, hkv, G, d = [40, 17], [5, 17], 2, 3, 64
    c = Cache(rng, S, hkv=hkv, d=d, dtype="f32")
    q = rng.standard_normal((sum(n), hkv * G, d))
    k, _, w, o = c.numpy()
    sinks = rng.standard_normal(hkv * G)
    qs = q_start_of(n)
    rows = [3, 17]
    nw, no, tol = bounded.key_weights(q, k, w, o, c.block_tables, S, qs, num_rows=rows, num_tokens=[100, 17],
                                      sinks=sinks, decay=0.5)
    for i in range(2):
        slots = [(c.block_tables[i][t // 16], t % 16) for t in range(S[i])]
        for g in range(hkv):
            keys = np.stack([k[b, g, :, s, :].reshape(-1) for b, s in slots])
            total = np.zeros(S[i])
            for j in range(rows[i]):
                for h in range(g * G, (g + 1) * G):
                    x = torch.as_tensor(keys @ q[qs[i] + j, h] / 8.0)
                    x[S[i] - n[i] + j + 1:] = -np.inf
                    x = torch.cat([x, torch.tensor([sinks[h]], dtype=torch.float64)])
                    total += torch.softmax(x, 0)[:-1].numpy()
            for t, (b, s) in enumerate(slots):
                new = t >= S[i] - n[i]
                assert abs(nw[b, g, s] - total[t] - (0 if new else 0.5 * w[b, g, s])) < 1e-12
                assert no[b, g, s] == ([100, 17][i] - S[i] + t if new else o[b, g, s])
                assert 0 < tol[b, g, s] < 1e-3


def test_evict_plan_by_hand():
    # one head, two blocks, 20 keys of which 8 stay
    w = np.zeros((2, 1, 16))
    w[1, 0, :16] = [5, 1, 9, 1, 0, 0, 0, 0, 7, 7, 7, 2, 0, 0, 0, 0]
    w[0, 0, :4] = [3, 7, 0, 0]
    o = np.zeros((2, 1, 16), dtype=np.int32)
    o[1, 0] = np.arange(16)
    o[0, 0, :4] = [16, 17, 18, 19]
    src, lens = bounded.evict_plan(w, o, np.array([[1, 0]]), [20], 2, max_keys=8, keep_first=1, keep_recent=2,
                                   num_tokens=[20])
    # kept: slots 0 (first), 18, 19 (recent), then 2 (9), 8, 9, 10, 17 (7 each)
    assert lens.tolist() == [8]
    assert src[0, 0].tolist() == [0, 8, 2, 9, 10, 17, 18, 19]
    # the lower slots of equals: with one key fewer, 17 leaves
    src, _ = bounded.evict_plan(w, o, np.array([[1, 0]]), [20], 2, max_keys=7, keep_first=1, keep_recent=2)
    assert src[0, 0].tolist() == [0, 8, 2, 9, 10, 18, 19]


def test_compact_by_hand():
    c = Cache(np.random.default_rng(3), [20], hkv=1, d=64, dtype="f32")
    k, v, w, o = c.numpy()
    src = np.array([[[0, 8, 2, 9, 10, 17, 18, 19]]], dtype=np.int32)
    nk, nv, nw, no = bounded.kv_compact(k, v, w, o, c.block_tables, src, [8])
    at = lambda t: (c.block_tables[0][t // 16], 0, t % 16)
    for d, s in enumerate(src[0, 0]):
        assert nw[at(d)] == w[at(s)] and no[at(d)] == o[at(s)]
        b, t = at(d)[0], d % 16
        np.testing.assert_array_equal(nk[b, 0, :, t], k[at(s)[0], 0, :, s % 16])
        np.testing.assert_array_equal(nv[b, 0, :, t], v[at(s)[0], 0, :, s % 16])
    # slots behind the eight are as they were
    np.testing.assert_array_equal(nw[c.block_tables[0][0], 0, 8:], w[c.block_tables[0][0], 0, 8:])
