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


def _groups(seed, count, most):
    """`count` groups of up to `most` requests; prefixes of up to 130 keys, two of them
    longer, one a later group's; some groups empty, some prefixes below a block."""
    rng = np.random.default_rng(seed)
    sizes = rng.integers(0, most + 1, size=count)
    sizes[[0, count // 2, count - 2]] = 1
    prefix = rng.integers(0, 131, size=count)
    prefix[[count // 2, count - 2]] = 1100, 390
    S, n = [], []
    for k in range(count):
        for _ in range(sizes[k]):
            n.append(int(rng.integers(0, 4)))
            # now and then fewer keys than the prefix
            S.append(max(n[-1], int(prefix[k] * rng.choice([1.0, 1.0, 0.6])) + int(rng.integers(0, 50))))
    lead = int(rng.integers(0, 3))
    for _ in range(lead + 2):
        S.append(int(rng.integers(3, 90)))
        n.append(2)
    return list(zip(sizes.tolist(), prefix.tolist())), S[-lead - 2:len(S) - 2] + S[:-lead - 2] + S[-2:], \
        n[-lead - 2:len(n) - 2] + n[:-lead - 2] + n[-2:], lead


@pytest.mark.parametrize("dtype,hq,hkv", [("bf16", 4, 2), ("f32", 3, 1)])
@pytest.mark.parametrize("count,most,inlined", [
    (64, 1, True), (65, 2, True), (130, 1, True), (200, 1, False), (130, 3, False), (300, 2, False),
    (2047, 1, False), (2048, 1, False), (2049, 1, False), (2200, 2, False)])
def test_many_groups(count, most, inlined, dtype, hq, hkv):
    """More groups than a wavefront has lanes, than a workgroup counts itself and than the
    schedule keeps in LDS, with items and rows that are numbered across such runs."""
    groups, S, n, lead = _groups(count + most, count, most)
    assert (count + len(S) <= 256) == inlined
    b = SharedBatch(count, groups, S, n, hq=hq, hkv=hkv, d=64, dtype=dtype, lead=lead, sinks=True, wide=True)
    args = b.to(DEV)
    got = b.call(DEV, args)
    b.check(got, "%d groups" % count)
    # whatever the workspace held
    size = av.attention_shared_workspace_size(args[0], args[1], args[3], num_groups=count, **b.bounds)
    assert size > 0
    again = b.call(DEV, args, workspace=torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV))
    assert torch.equal(again, got)
