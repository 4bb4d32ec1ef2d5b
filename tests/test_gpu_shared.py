"""verify_attention_shared against the oracle."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
from bounded_common import bits
from shared_common import SharedBatch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

CASES = [
    # groups (requests, prefix), S, n, options
    ("one", [(1, 16)], [17], [1], {}),
    ("two", [(2, 333)], [360, 345], [1, 9], {}),
    ("exact", [(3, 64)], [64, 65, 80], [1, 1, 16], {}),                       # a request that is all prefix
    ("many", [(20, 200)], [210 + 13 * i for i in range(20)], [1] * 20, {}),
    ("verify", [(8, 400)], [420 + 31 * i for i in range(8)], [9] * 8, {}),
    ("kinds", [(3, 130), (1, 700), (2, 15), (0, 50), (4, 48)], [150, 400, 131, 800, 40, 16, 60, 49, 333, 64],
     [5, 17, 1, 3, 2, 16, 1, 1, 9, 2], dict(lead=0, sinks=True)),
    ("apart", [(2, 100)], [50, 120, 130, 77, 1], [3, 2, 0, 5, 1], dict(lead=1)),  # requests of no group, one without rows
    ("inside", [(3, 320)], [330, 325, 320], [40, 200, 320], {}),                # rows that stand inside the prefix
    ("prompts", [(3, 512)], [512 + 100, 512 + 333, 512 + 1], [100, 333, 1], {}),  # prompts behind the prefix
    ("rows", [(5, 96)], [120, 111, 130, 140, 100], [3, 7, 2, 5, 4], {}),
    ("unmapped", [(3, 160)], [200, 180, 260], [4, 9, 2], dict(unmapped=[(0, 2), (1, 2), (2, 2), (2, 12), (1, 11)])),
    ("longer than cached", [(2, 400), (2, 90)], [130, 120, 50, 95], [3, 40, 2, 5], {}),  # prefixes beyond the keys
    ("spikes", [(4, 1000)], [1100, 1030, 2000, 1001], [2, 3, 4, 1], dict(spike=True)),
    ("no prefix", [(2, 0), (2, 40)], [70, 30, 50, 90], [2, 3, 1, 4], {}),
]
HEADS = [(8, 2, 128, "bf16"), (8, 1, 64, "bf16"), (10, 2, 128, "bf16"), (8, 2, 128, "f32"), (3, 3, 64, "f32"), (16, 1, 64, "f32")]


@pytest.mark.parametrize("hq,hkv,d,dtype", HEADS)
@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("name,groups,S,n,opt", CASES, ids=[c[0] for c in CASES])
def test_shared(name, groups, S, n, opt, wide, hq, hkv, d, dtype):
    b = SharedBatch(len(S) + hq, groups, S, n, hq=hq, hkv=hkv, d=d, dtype=dtype, wide=wide, **opt)
    args = b.to(DEV)
    before = [t.clone() for t in args]
    got = b.call(DEV, args)
    b.check(got, name)
    for x, y in zip(args, before):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # the same call gives the same bits, whatever its workspace and output held
    size = av.attention_shared_workspace_size(args[0], args[1], args[3], num_groups=len(groups), **b.bounds)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full_like(got, float("nan"))
    assert b.call(DEV, args, workspace=ws, out=out) is out
    np.testing.assert_array_equal(bits(out), bits(got))


@pytest.mark.parametrize("short,long", [(1, 18), (1, 24), (3, 50), (17, 20)])
@pytest.mark.parametrize("keys", [1, 20, 140, 500, 1300])
def test_rows_of_very_different_numbers_share_few_units(short, long, keys):
    """Ranges of a few units, in which the rows' tiles weigh differently."""
    n = [short, long, short]
    b = SharedBatch(keys + long, [(3, 32)], [32 + keys + long, 32 + keys + long, 40 + short], n, hq=8, hkv=1, d=64,
                    dtype="bf16", wide=True)
    b.check(b.call(DEV))


@pytest.mark.parametrize("dtype,d,n", [("f32", 128, [130] * 3), ("bf16", 128, [700, 650]), ("bf16", 64, [900, 850])])
def test_a_prefix_of_more_row_tiles_than_workgroups_are_left_for_the_requests(dtype, d, n):
    """The requests' partial results are numbered without the prefixes'."""
    S = [p + 16 + 20 * i for i, p in enumerate(n)]
    b = SharedBatch(7, [(len(n), 16)], S, n, hq=32, hkv=4, d=d, dtype=dtype)
    b.check(b.call(DEV, max_seq_len=16 * b.table.shape[1]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_prefix_and_long_requests(dtype):
    n = [1 + i % 6 for i in range(24)]
    b = SharedBatch(5, [(20, 4100)], [4100 + 61 * i + n[i] for i in range(24)], n, hq=8, hkv=2, d=128, dtype=dtype, sinks=True)
    b.check(b.call(DEV))


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("batch", [511, 512, 700])
def test_more_requests_than_a_workgroup_counts_itself(batch, wide):
    rng = np.random.default_rng(batch)
    sizes = [batch // 3, 0, batch // 2]
    lens = [int(x) for x in rng.integers(49, 120, size=batch)]
    n = [int(x) for x in rng.integers(0, 4, size=batch)]
    b = SharedBatch(batch, list(zip(sizes, [32, 10, 48])), lens, n, hq=4, hkv=2, d=64, dtype="bf16", lead=2, wide=wide)
    b.check(b.call(DEV))


@pytest.mark.parametrize("keys,dtype,d,short", [
    (2048, "bf16", 128, True), (2049, "bf16", 128, False), (4096, "bf16", 64, True), (4097, "bf16", 64, False),
    (448, "f32", 128, True), (449, "f32", 128, False), (704, "f32", 64, True), (705, "f32", 64, False)])
def test_short_requests_need_no_workspace(keys, dtype, d, short):
    """On both sides of the longest short request, with more rows than one tile and than
    max_q_len."""
    n = [1, 9, 30]
    b = SharedBatch(keys, [(2, 333)], [keys, 340, keys - 50], n, hq=10, hkv=2, d=d, dtype=dtype, sinks=True)
    args = b.to(DEV)
    assert (av.attention_shared_workspace_size(args[0], args[1], args[3], num_groups=1, **b.bounds) == 0) == short
    b.check(b.call(DEV, args))
    b.check(b.call(DEV, args, max_q_len=2))


@pytest.mark.parametrize("wide", [False, True])
def test_bounds_that_are_not_tight_and_a_request_beyond_max_q_len(wide):
    b = SharedBatch(3, [(3, 200)], [260, 300, 210], [3, 70, 2], hq=8, hkv=2, d=128, dtype="bf16", wide=wide)
    for kw in (dict(max_q_len=1), dict(max_q_len=500), dict(max_seq_len=16 * b.table.shape[1]), dict(max_prefix_len=5000)):
        b.check(b.call(DEV, **kw), str(kw))
    # a smaller bound cuts the shared part, not the result
    b.check(b.call(DEV, max_prefix_len=100))
    # without groups, or with prefixes below a block, the call is verify_attention
    q, k, v, table, S, qs, gs, pl = b.to(DEV)
    v = torch.nan_to_num(v, nan=0.0)
    k = torch.nan_to_num(k, nan=0.0)
    bounds = dict(max_q_len=70, max_seq_len=300)
    want = av.verify_attention(q, k, v, table, S, qs, **bounds)
    for g, p, m in ((gs[:1], pl[:0], 200), (gs, pl, 15)):
        got = av.verify_attention_shared(q, k, v, table, S, qs, g, p, max_prefix_len=m, **bounds)
        np.testing.assert_array_equal(bits(got), bits(want))


@pytest.mark.parametrize("wide", [False, True])
def test_rows_behind_the_last_request_stay_as_they_were(wide):
    b = SharedBatch(9, [(2, 64)], [80, 90], [2, 3], hq=4, hkv=2, d=64, dtype="bf16", wide=wide)
    q, *rest = b.to(DEV)
    q = torch.cat([q, q[:2]])
    out = torch.full_like(q, 7.0)
    b.call(DEV, [q] + rest, out=out)
    b.check(out[:5])
    assert (out[5:] == 7).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_operands_at_odd_addresses(dtype, wide):
    """q and out need only be aligned to an element."""
    b = SharedBatch(2, [(3, 100)], [150, 120, 300], [4, 1, 9], hq=8, hkv=2, d=128, dtype=dtype, wide=wide)
    args = b.to(DEV)
    want = b.call(DEV, args)
    flat = torch.zeros(args[0].numel() + 3, dtype=args[0].dtype, device=DEV)
    q, out = flat[3:].view(args[0].shape), torch.zeros_like(flat)[1:-2].view(args[0].shape)
    q.copy_(args[0])
    np.testing.assert_array_equal(bits(b.call(DEV, [q] + args[1:], out=out)), bits(want))


@pytest.mark.parametrize("wide", [False, True])
def test_captured_and_replayed_on_new_lengths(wide):
    """A graph's launch holds for any lengths within its bounds."""
    b = SharedBatch(4, [(3, 320)], [500, 400, 350], [4, 2, 9], hq=8, hkv=2, d=64, dtype="bf16", sinks=True, wide=wide)
    args = b.to(DEV)
    sinks = b.sinks.to(DEV)
    bounds = dict(max_q_len=9, max_seq_len=4160 if wide else 600, max_prefix_len=400)
    ws = torch.empty(av.attention_shared_workspace_size(args[0], args[1], args[3], num_groups=1, **bounds),
                     dtype=torch.uint8, device=DEV)
    out = torch.empty_like(args[0])
    run = lambda o, w: av.verify_attention_shared(*args, sinks=sinks, out=o, workspace=w, **bounds)
    run(out, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(out, ws)
    for prefix, shorter in ((320, 0), (100, 1), (0, 3), (333, 2)):
        args[7].fill_(prefix)
        args[4].copy_(torch.as_tensor(b.S - shorter))
        g.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(bits(out), bits(run(None, None)))


@pytest.mark.parametrize("wide", [False, True])
def test_two_calls_at_once_on_streams_of_their_own(wide):
    b = [SharedBatch(s, [(6, 640)], [700 + 50 * i for i in range(6)], [5] * 6, hq=8, hkv=2, d=128, dtype="bf16", wide=wide)
         for s in (1, 2)]
    args = [x.to(DEV) for x in b]
    want = [bits(x.call(DEV, a)) for x, a in zip(b, args)]
    streams = [torch.cuda.Stream() for _ in b]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [x.call(DEV, a, stream=s) for x, a, s in zip(b, args, streams)]
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            np.testing.assert_array_equal(bits(g), w)
