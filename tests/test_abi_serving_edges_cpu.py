"""Bounds of the serving calls at their exact values, on the host."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
from test_abi_bounded_cpu import DUMMY, _attn
from test_abi_serving_cpu import _adjust, _count


@pytest.mark.parametrize("vocab,want", [(2 ** 31 - 33, av.EINVAL), (2 ** 31 - 32, av.EUNSUPPORTED), (2 ** 31, av.EUNSUPPORTED)])
def test_count_tokens_refuses_vocabularies_from_the_stated_one_on(vocab, want):
    """The last one that is taken is refused for its missing tokens, nothing else."""
    assert _count(V=vocab, tokens=None) == want


@pytest.mark.parametrize("vocab,want", [(2 ** 31 - 2050, av.EINVAL), (2 ** 31 - 2049, av.EUNSUPPORTED)])
def test_adjust_logits_refuses_vocabularies_from_the_stated_one_on(vocab, want):
    assert _adjust(V=vocab, logits=None) == want


@pytest.mark.parametrize("batch,want", [(65535, av.EINVAL), (65536, av.EUNSUPPORTED)])
def test_requests(batch, want):
    assert _count(B=batch, tokens=None) == want
    assert _adjust(B=batch, logits=None) == want


def _groups(params=True, ms=100, G=2, mp=64, gs=DUMMY, pl=DUMMY, lens=DUMMY, bt=DUMMY, counts=DUMMY, **kw):
    p = _attn(**kw)
    return av.library().verify_check_groups(ctypes.byref(p) if params else None, ms, G, mp, gs, pl, lens, bt, counts, None)


@pytest.mark.parametrize("kw,want", [
    (dict(params=False), av.EINVAL), (dict(counts=None), av.EINVAL), (dict(ms=-1), av.EINVAL), (dict(G=-1), av.EINVAL),
    (dict(mp=-1), av.EINVAL), (dict(num_seqs=-1), av.EINVAL), (dict(block_size=32), av.EINVAL),
    (dict(max_blocks_per_seq=0), av.EINVAL), (dict(G=65536), av.EUNSUPPORTED), (dict(num_seqs=65536), av.EUNSUPPORTED),
    (dict(gs=None), av.EINVAL), (dict(pl=None), av.EINVAL), (dict(lens=None), av.EINVAL), (dict(bt=None), av.EINVAL),
])
def test_check_groups(kw, want):
    assert _groups(**kw) == want


def test_the_binding_refuses_groups():
    i32 = torch.int32
    good = [torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(4, dtype=i32), torch.zeros((4, 5), dtype=i32)]
    bounds = dict(max_prefix_len=16, max_seq_len=80)
    for at, t in [(0, good[0][:0]), (0, good[3]), (0, good[0].long()), (1, good[1][:1]), (2, good[2][:3]), (3, good[3][0]),
                  (3, good[3][:, :0]), (3, good[3].float()), (0, good[0])]:
        args = list(good)
        args[at] = t
        with pytest.raises((ValueError, TypeError)):
            av.check_groups(*args, **bounds)


def test_axes_of_any_kind_name_the_same_frequencies():
    """A layer's parameters are kept by what the axes say, not by how they are given: a
    tensor of one axis is a number too."""
    q, freq = torch.zeros((2, 1, 64)), torch.ones(1, dtype=torch.float64)
    pos = torch.zeros((3, 2), dtype=torch.int32)
    for axes in (torch.tensor([2]), (0,), np.array([1]), [1], torch.tensor([1]), (2,), np.array([0], dtype=np.uint8), [0.0],
                 range(1, 2), b"\2"):
        params, _, _ = av._rotary_args(q, 2, 64, pos, freq, axes, False, 0.0, -1, q.device)
        assert list(params.axis[:1]) == [int(axes[0])]
    freq = torch.ones(3, dtype=torch.float64)
    for axes in (torch.tensor([2, 0, 1]), (0, 0, 2), np.array([1, 2, 0]), [0.0, 1.0, 2.0], range(3)):
        params, _, _ = av._rotary_args(q, 2, 64, pos, freq, axes, False, 0.0, -1, q.device)
        assert list(params.axis[:3]) == [int(x) for x in axes]
    for axes in ((3,), (-1,), (300,), torch.tensor([3]), np.array([-1], dtype=np.int8)):
        with pytest.raises(ValueError, match="axes"):
            av._rotary_args(q, 2, 64, pos, freq[:1], axes, False, 0.0, -1, q.device)
