"""verify_attention_shared at the ends of its ranges: row tiles by the ten thousand with
hardly a key, and groups by the hundred and the thousand."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
from shared_common import SharedBatch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("max_seq_len", [0, 5])
def test_more_row_tiles_than_a_launch_has_in_z(max_seq_len):
    """33000 rows of 32 heads are 66000 tiles of 16 rows; at so few keys they are walked
    by the launch for short requests.  Only the last rows see a key."""
    rows, keys = 33000, 5
    b = SharedBatch(1, [(1, 16)], [keys], [keys], hq=32, hkv=1, d=64, dtype="bf16")
    q, k, v, table, S, _, gs, pl = b.to(DEV)
    many = torch.randn((rows, 32, 64), device=DEV).to(q.dtype)
    many[rows - keys:] = q
    bounds = dict(max_q_len=rows, max_seq_len=max_seq_len, max_prefix_len=16)
    assert av.attention_shared_workspace_size(many, k, table, num_groups=1, **bounds) == 0
    out = torch.full_like(many, 7.0)
    q_start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    av.verify_attention_shared(many, k, v, table, S, q_start, gs, pl, out=out, **bounds)
    seen = min(max_seq_len, keys)
    assert (out[:rows - seen] == 0).all()
    if seen:
        b.check(out[rows - keys:])
