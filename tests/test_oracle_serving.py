"""Pins of the oracle's head norms, changed logits and token counts."""
from __future__ import annotations

import numpy as np

from oracle import serving


def test_a_normed_head_has_its_weights_length():
    x = np.random.default_rng(0).standard_normal((5, 3, 64)) * 7
    y = serving.head_norm(x, None, 0.0)
    np.testing.assert_allclose((y * y).sum(-1), 64.0, rtol=1e-12)
    w = np.arange(64.0)
    np.testing.assert_allclose(serving.head_norm(x, w, 0.0), y * w, rtol=1e-12)
    # a factor of the head is taken out again, and eps bounds what an empty head becomes
    np.testing.assert_allclose(serving.head_norm(x * 1e3, None, 0.0), y, rtol=1e-12)
    assert not serving.head_norm(np.zeros((1, 1, 64)), None, 1e-6).any()


def test_words_hold_the_lowest_bit_first():
    t = np.zeros(40, dtype=bool)
    t[[0, 31, 33]] = True
    np.testing.assert_array_equal(serving.words(t).view(np.uint32), [0x80000001, 2])
    np.testing.assert_array_equal(serving.bits(serving.words(t), 40), t)


def test_adjusted_logits_by_hand():
    x = np.array([[2.0, -2.0, 4.0, 1.0, -1.0]] * 3)
    counts, seen = np.array([[0, 3, 0, 0, 0]]), np.zeros((1, 2, 1), dtype=np.int32)
    seen[0, 0, 0], seen[0, 1, 0] = 1, 2  # token 0 in the prompt, token 1 put out three times
    y, _, touched = serving.adjust_logits(
        x, np.array([4, 2, 2]), [0, 3], counts=counts, seen=seen, repetition=[2.0], frequency=[0.5], presence=[0.25],
        bias_start=[0, 3], bias_tokens=[3, 3, 9], bias_values=[1.0, 0.5, 7.0],
        mask=np.array([[0b10111]], dtype=np.int32), mask_rows=[-1, 0, 5])
    np.testing.assert_array_equal(y[0], [1.0, -4 - 1.5 - 0.25, 4.0, 2.5, -1.0])
    np.testing.assert_array_equal(y[1], [1.0, -5.75, 2 - 0.5 - 0.25, -np.inf, -1.0])  # the draft 2 counts
    np.testing.assert_array_equal(y[2], [1.0, -5.75, 2 - 1.0 - 0.25, 2.5, -1.0])      # twice; no such mask
    np.testing.assert_array_equal(touched[0], [True, True, False, True, False])


def test_counted_tokens_by_hand():
    counts, seen = np.zeros((2, 35), dtype=np.int32), np.zeros((2, 2, 2), dtype=np.int32)
    c, s = serving.count_tokens(counts, seen, [3, 3, -1, 34, 7, 99], [0, 4, 6], num=[3, 2], slots=[1, 0])
    assert c[1, 3] == 2 and c[1, 34] == 0 and c[0, 7] == 1 and c.sum() == 3
    assert s[1, 1, 0] == 8 and s[0, 1, 0] == 128 and not s[:, 0].any()
    c, s = serving.count_tokens(counts, seen, [34], [0, 1, 1], prompt=True)
    assert not c.any() and s[0, 0, 1] == 4 and not s[:, 1].any()
