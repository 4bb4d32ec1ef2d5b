"""verify_check_groups against a host restatement, on batches whose groups are right and on
seeded corruptions of them; and what check=True refuses of the serving calls."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
from bounded_common import bits
from shared_common import SharedBatch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def host_check(group_start, prefix, S, table, max_prefix_len, max_seq_len):
    G, B = len(prefix), len(S)
    bounds = [k for k in range(G) if group_start[k] < 0 or group_start[k + 1] < group_start[k] or group_start[k + 1] > B]
    bad, first = [], list(bounds)
    cached = np.clip(S, 0, min(max_seq_len, 16 * table.shape[1]))
    for i in range(B):
        k = int(np.searchsorted(group_start[:G], i, side="right")) - 1
        if k < 0 or not i < group_start[k + 1]:
            continue
        r = max(int(group_start[k]), 0)
        blocks = min(max(0, min(int(prefix[k]), max_prefix_len, int(cached[r]))) // 16, -(-int(cached[i]) // 16))
        if (table[i, :blocks] != table[r, :blocks]).any():
            bad.append(i)
            first.append(k)
    return {"bounds": len(bounds), "table": len(bad)}, min(first, default=-1)


def both(gs, prefix, S, table, **bounds):
    dev = [torch.as_tensor(np.asarray(x, dtype=np.int32)).to(DEV) for x in (gs, prefix, S, table)]
    got = av.check_groups(*dev, **bounds)
    assert got == host_check(np.asarray(gs), prefix, S, np.asarray(table), **bounds)
    return got


def batch(**kw):
    return SharedBatch(6, [(3, 130), (0, 40), (4, 48), (2, 15)], [60, 150, 400, 131, 49, 60, 333, 64, 40, 16, 9],
                       [3, 5, 17, 1, 2, 1, 9, 2, 1, 3, 2], hq=4, hkv=2, d=64, dtype="bf16", lead=1, **kw)


def test_against_the_host():
    b = batch()
    limits = dict(max_prefix_len=130, max_seq_len=400)
    assert both(b.group_start, b.prefix, b.S, b.table, **limits) == ({"bounds": 0, "table": 0}, -1)
    table = b.table.copy()
    table[2, 7] += 1    # the prefix's last whole block
    table[6, 3] += 1    # behind the prefix: the request's own
    table[10, 0] += 1   # of no group
    table[9, 0] += 1    # a prefix below a block
    table[0, 0] += 1
    assert both(b.group_start, b.prefix, b.S, table, **limits) == ({"bounds": 0, "table": 1}, 0)
    assert both(b.group_start, b.prefix, b.S, table, max_prefix_len=120, max_seq_len=400)[1] == -1  # not shared any more
    S = b.S.copy()
    S[2] = 112          # the request has no key there
    assert both(b.group_start, b.prefix, S, table, **limits)[1] == -1
    table[4, 0] += 1    # a group's first request: the others differ from it
    assert both(b.group_start, b.prefix, b.S, table, **limits) == ({"bounds": 0, "table": 4}, 0)
    for at, value, count in ((4, 12, 1), (0, -1, 1), (2, 1, 1), (1, 11, 1)):
        gs = b.group_start.copy()
        gs[at] = value
        dev = [torch.as_tensor(x).to(DEV) for x in (gs, b.prefix, b.S, b.table)]
        assert av.check_groups(*dev, **limits)[0]["bounds"] == count
    rng = np.random.default_rng(0)
    for _ in range(40):  # sorted and not, of any values
        gs = rng.integers(-2, 14, size=5)
        gs = np.sort(gs) if rng.random() < 0.7 else gs
        t = np.where(rng.random(b.table.shape) < 0.02, -1, b.table[0])
        if np.all(np.diff(gs) >= 0):
            both(gs, rng.integers(-5, 200, size=4), b.S, t, max_prefix_len=int(rng.integers(0, 200)), max_seq_len=300)
        else:  # where a request's group is sought in an unsorted list is not stated: no fault
            dev = [torch.as_tensor(np.asarray(x, dtype=np.int32)).to(DEV) for x in (gs, b.prefix, b.S, t)]
            assert av.check_groups(*dev, max_prefix_len=100, max_seq_len=300)[0]["bounds"] > 0


def test_many_groups_and_requests():
    B, G = 9000, 5000
    rng = np.random.default_rng(1)
    gs = np.sort(rng.integers(0, B + 1, size=G + 1)).astype(np.int32)
    k = np.searchsorted(gs[:G], np.arange(B), side="right") - 1
    table = np.stack([k * 2, k * 2 + 1, 100000 + np.arange(B)], axis=1)
    limits = dict(max_prefix_len=32, max_seq_len=48)
    assert both(gs, np.full(G, 32), np.full(B, 48), table, **limits)[0] == {"bounds": 0, "table": 0}
    members = [i for i in range(B) if k[i] >= 0 and i > gs[k[i]]]
    for i in (members[0], members[-1], members[len(members) // 2]):
        table[i, 1] = -7
    assert both(gs, np.full(G, 32), np.full(B, 48), table, **limits) == ({"bounds": 0, "table": 3}, int(k[members[0]]))


@pytest.mark.parametrize("wide", [False, True])
def test_shared_attention_refuses_bad_groups_before_launching(wide):
    b = batch(wide=wide)
    args = b.to(DEV)
    out = torch.full_like(args[0], 7.0)
    want = b.call(DEV, args)
    np.testing.assert_array_equal(bits(b.call(DEV, args, check=True)), bits(want))
    for at, place, value, kind, first in ((3, (2, 1), int(args[3][2, 2]), "table", 0), (6, 3, 1, "bounds", 2)):
        bad = [t.clone() for t in args]
        bad[at][place] = value
        with pytest.raises(av.BatchError, match="first group %d" % first) as e:
            b.call(DEV, bad, out=out, check=True)
        assert e.value.counts[kind] >= 1 and e.value.first == first
        torch.cuda.synchronize()
        assert (out == 7).all()
    # the batch's own descriptor is checked first
    bad = [t.clone() for t in args]
    bad[3][5, 0] = -1
    with pytest.raises(av.BatchError, match="first request 5") as e:
        b.call(DEV, bad, out=out, check=True)
    assert e.value.counts["block_id"] == 1 and (out == 7).all()


def test_norms_and_changed_logits_refuse_a_bad_batch_before_launching():
    b = batch()
    q, k, v, table, S, qs, *_ = b.to(DEV)
    T = q.shape[0]
    new = torch.ones((T, 2, 64), dtype=q.dtype, device=DEV)
    pos, freq = torch.zeros(T, dtype=torch.int32, device=DEV), torch.ones(32, dtype=torch.float64, device=DEV)
    before = bits(k).copy(), bits(v).copy()
    bad_table = table.clone()
    bad_table[3, (int(b.S[3]) - 1) // 16] = b.nb
    out = torch.full_like(q, 7.0)
    with pytest.raises(av.BatchError, match="verify_norm_rotary_append") as e:
        av.verify_norm_rotary_append(q, new, new, pos, freq, k, v, bad_table, S, qs, q_out=out, check=True)
    assert e.value.counts["block_id"] == 1 and e.value.first == 3 and (out == 7).all()
    np.testing.assert_array_equal(bits(k), before[0])
    np.testing.assert_array_equal(bits(v), before[1])
    want = av.verify_norm_rotary_append(q, new, new, pos, freq, k.clone(), v.clone(), table, S, qs)
    np.testing.assert_array_equal(
        bits(av.verify_norm_rotary_append(q, new, new, pos, freq, k, v, table, S, qs, check=True)), bits(want))
    x, tok = torch.randn((T, 70), device=DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
    mask, rows = torch.full((1, 3), 5, dtype=torch.int32, device=DEV), torch.zeros(T, dtype=torch.int32, device=DEV)
    y = torch.full_like(x, 7.0)
    short = qs.clone()
    short[-1] -= 1
    with pytest.raises(av.BatchError, match="verify_adjust_logits") as e:
        av.verify_adjust_logits(x, tok, short, mask=mask, mask_rows=rows, out=y, check=True)
    assert e.value.counts["rows"] == 1 and e.value.first == len(b.S) - 1 and (y == 7).all()
    got = av.verify_adjust_logits(x, tok, qs, mask=mask, mask_rows=rows, out=y, check=True)
    assert torch.isfinite(got).sum() == 6 * T  # two bits of each of three words
