"""Bounds of the serving calls at their exact values, on the host."""
from __future__ import annotations

import pytest

import paper_2608_24004_amd as av
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
