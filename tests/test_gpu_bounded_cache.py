"""verify_key_weights, verify_evict_plan and verify_kv_compact against the oracle, and
the calls of a bounded cache together."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
import workload
from bounded_common import BLOCK, Cache, bits, q_start_of
from oracle import bounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(x, dtype=torch.int32):
    return None if x is None else torch.as_tensor(np.asarray(x), dtype=dtype, device=DEV)


def _weights_case(rng, S, n, hkv, G, d, dtype, *, rows=None, lost=None, sinks=False, decay=1.0, unmapped=0, size=1.0,
                  max_q_len=None, max_seq_len=None):
    c = Cache(rng, S, hkv=hkv, d=d, dtype=dtype, unmapped=unmapped, lost=lost)
    qs = q_start_of(n)
    q = torch.as_tensor(size * rng.standard_normal((int(qs[-1]), hkv * G, d))).to(workload.torch_dtype(dtype))
    sk = rng.standard_normal(hkv * G).astype(np.float32) if sinks else None
    tokens = None if lost is None else c.tokens
    kc, _, w, o, bt, sl = c.to(DEV)
    bounds = dict(max_q_len=max(n) if max_q_len is None else max_q_len,
                  max_seq_len=max(S) if max_seq_len is None else max_seq_len)
    got = av.verify_key_weights(q.to(DEV), kc, w, o, bt, sl, _dev(qs), num_rows=_dev(rows), num_tokens=_dev(tokens),
                                sinks=_dev(sk, torch.float32), decay=decay, **bounds)
    torch.cuda.synchronize()
    assert got.data_ptr() == w.data_ptr()
    k, _, w0, o0 = c.numpy()
    S_used = np.minimum(S, bounds["max_seq_len"])
    rw, ro, tol = bounded.key_weights(q.double().numpy(), k, w0, o0, c.block_tables, S_used, qs, num_rows=rows,
                                      num_tokens=tokens if tokens is not None else None, sinks=sk, decay=decay)
    np.testing.assert_array_equal(o.cpu().numpy(), ro)
    gw = w.double().cpu().numpy()
    same = np.isnan(rw)
    np.testing.assert_array_equal(np.isnan(gw), same)  # slots of no key are as they were
    off = np.abs(gw - rw)
    assert (off[~same] <= tol[~same]).all(), "worst %.3g of its tolerance" % np.nanmax(off / np.maximum(tol, 1e-300))


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("S,n,hkv,G,kw", [
    ([1], [1], 1, 1, {}),
    ([1501], [1], 2, 4, {}),
    ([15, 16, 17, 64, 65], [1, 2, 3, 5, 9], 2, 4, dict(rows=[1, 0, 2, 5, 4])),
    ([300, 0, 33, 129], [9, 0, 33, 0], 1, 5, dict(lost=[100, 0, 0, 7], decay=0.5)),
    ([70, 150], [70, 150], 1, 2, dict(sinks=True)),              # whole prompts
    ([260, 31, 5], [40, 31, 5], 1, 8, dict(rows=[37, 1, 9])),    # more rows than one staging holds
    ([140, 31], [15, 9], 2, 8, {}),                              # eight row tiles, all in one workgroup
    ([140, 31], [9, 16], 1, 16, {}),                             # ten, in two even parts
    ([900], [300], 1, 4, dict(rows=[299])),                      # rows in segments
    ([700, 400], [300, 20], 1, 4, dict(max_q_len=130)),          # segments, and more rows than announced
    ([30, 40], [0, 0], 2, 4, dict(decay=0.75, max_q_len=3)),     # no row at all
    ([200, 90], [5, 17], 2, 1, dict(unmapped=3, decay=0.0)),
    ([400, 37], [6, 20], 1, 8, dict(size=15.0, sinks=True)),     # peaked rows
    ([100, 80], [30, 40], 2, 8, dict(max_q_len=2)),              # more rows than announced
    ([100, 80], [3, 4], 1, 2, dict(max_seq_len=81)),             # more keys than announced
    ([300, 90, 33, 0], [1, 3, 0, 1], 2, 3, dict(max_q_len=1)),   # one row: its scores; more: its keys again
    ([200, 90], [1, 1], 1, 2, dict(rows=[0, 1], unmapped=4, sinks=True)),
    ([700, 1, 2, 17], [1, 1, 1, 1], 1, 1, {}),                   # bounds well beyond what the cache holds
])
def test_key_weights(d, dtype, S, n, hkv, G, kw):
    _weights_case(np.random.default_rng(len(S) * d + G), S, n, hkv, G, d, dtype, **kw)


@pytest.mark.parametrize("S,n,kw", [([5000, 40], [2, 1], {}), ([2600], [150], {}), ([2500, 2300], [7, 5], dict(decay=0.25)),
                                    ([9000, 4100], [1, 1], dict(decay=0.25, unmapped=5)), ([3000], [2], {})])
def test_key_weights_of_long_caches(S, n, kw):
    _weights_case(np.random.default_rng(sum(S)), S, n, 1, 4, 128, "bf16", **kw)


def test_key_weights_give_the_same_bits_again():
    rng = np.random.default_rng(8)
    S, n = [700, 90, 333], [9, 3, 1]
    c = Cache(rng, S, hkv=2, d=128, dtype="bf16")
    q = torch.randn((sum(n), 8, 128), device=DEV).to(torch.bfloat16)
    outs = []
    for _ in range(3):
        kc, _, w, o, bt, sl = c.to(DEV)
        av.verify_key_weights(q, kc, w, o, bt, sl, _dev(q_start_of(n)), max_q_len=9, max_seq_len=700)
        outs.append(bits(w))
    np.testing.assert_array_equal(outs[0], outs[1])
    np.testing.assert_array_equal(outs[0], outs[2])


def test_key_weights_not_finite():
    """A NaN key makes the weights of its rows' keys NaN, as the softmax does, those of
    the other requests and of keys that no such row sees not; an infinite key that
    scores -inf weighs nothing."""
    rng = np.random.default_rng(9)
    S, n = [40, 40], [1, 2]
    c = Cache(rng, S, hkv=1, d=64, dtype="f32")
    kc, _, w, o, bt, sl = c.to(DEV)
    q = torch.ones((3, 1, 64), device=DEV)
    at = lambda i, t: (int(c.block_tables[i, t // 16]), 0, slice(None), t % 16)
    kc[at(1, 39)] = float("nan")      # seen by the second row of request 1 alone
    kc[at(0, 7)] = float("-inf")
    av.verify_key_weights(q, kc, w, o, bt, sl, _dev(q_start_of(n)), num_rows=_dev([1, 1]), max_q_len=2, max_seq_len=40,
                          decay=0.0)
    line = lambda i: torch.cat([w[int(b), 0] for b in c.block_tables[i]])[:40].cpu()
    assert torch.isfinite(line(0)).all() and line(0)[7] == 0 and abs(float(line(0).sum()) - 1) < 1e-5
    assert torch.isfinite(line(1)).all() and line(1)[39] == 0 and abs(float(line(1).sum()) - 1) < 1e-5
    av.verify_key_weights(q, kc, w, o, bt, sl, _dev(q_start_of(n)), max_q_len=2, max_seq_len=40, decay=0.0)
    assert torch.isfinite(line(0)).all()
    assert torch.isnan(line(1)).all()


def _plan_case(c, dw, do, *, max_keys, tokens, max_seq_len=None, **kw):
    _, _, _, _, bt, sl = c.to(DEV)
    src, lens = av.verify_evict_plan(dw, do, bt, sl, max_keys=max_keys, num_tokens=_dev(tokens),
                                     max_seq_len=int(c.S.max(initial=0)) if max_seq_len is None else max_seq_len, **kw)
    torch.cuda.synchronize()
    S = c.S if max_seq_len is None else np.minimum(c.S, max_seq_len)
    rs, rl = bounded.evict_plan(dw.double().cpu().numpy(), None if do is None else do.cpu().numpy(), c.block_tables, S,
                                c.nb, max_keys=max_keys, num_tokens=tokens, **kw)
    np.testing.assert_array_equal(lens.cpu().numpy(), rl)
    np.testing.assert_array_equal(src.cpu().numpy(), rs)
    return src, lens


def _plain_cache(rng, S, hkv, **kw):
    return Cache(rng, S, hkv=hkv, d=64, dtype="bf16", **kw)


@pytest.mark.parametrize("S,hkv,max_keys,kw", [
    ([1], 1, 1, {}),
    ([2], 1, 1, {}),
    ([100, 33, 0, 64, 65], 2, 64, dict(keep_first=4, keep_recent=16)),
    ([200, 150], 3, 16, dict(keep_first=8, keep_recent=8)),   # nothing left to weigh
    ([500], 2, 499, {}),
    ([500, 20], 2, 700, dict(keep_recent=9)),                 # nobody exceeds it
    ([333, 90], 1, 7, dict(keep_recent=1)),
])
@pytest.mark.parametrize("values", ["spread", "equal", "few", "odd"])
@pytest.mark.parametrize("lost", [False, True])
def test_evict_plan(S, hkv, max_keys, kw, values, lost):
    rng = np.random.default_rng(max_keys + len(S))
    c = _plain_cache(rng, S, hkv, lost=[3 * s for s in S] if lost else None)
    w = c.w.clone()
    if values == "equal":
        w = torch.zeros_like(w)
    elif values == "few":
        w = torch.as_tensor(rng.integers(0, 3, size=w.shape), dtype=torch.float32)
    elif values == "odd":
        w = torch.as_tensor(rng.choice([0.0, -0.0, 1.0, np.inf, -np.inf, np.nan, 1e-42, -1.0, 3e38], size=w.shape),
                            dtype=torch.float32)
    o = c.o.to(DEV) if lost else None
    _plan_case(c, w.to(DEV), o, max_keys=max_keys, tokens=c.tokens if lost else None, **kw)


@pytest.mark.parametrize("S,hkv", [([40000, 16385, 16384], 2), ([8193, 4097, 8192], 2), ([4097, 4096], 3),
                                   ([250000, 100, 170003], 1)])
def test_evict_plan_of_long_caches(S, hkv):
    """More blocks than the workgroup has threads, and ordinals that are none."""
    rng = np.random.default_rng(4)
    c = Cache.__new__(Cache)
    c.S = np.asarray(S, dtype=np.int32)
    blocks = -(-c.S // BLOCK)
    c.nb = int(blocks.sum())
    ids = rng.permutation(c.nb).astype(np.int32)
    c.block_tables = np.full((len(S), int(blocks.max())), -1, dtype=np.int32)
    for i, off in enumerate(np.cumsum(blocks) - blocks):
        c.block_tables[i, :blocks[i]] = ids[off:off + blocks[i]]
    c.k = c.v = torch.zeros(1)
    c.w = torch.as_tensor(rng.integers(0, 5000, size=(c.nb, hkv, BLOCK)), dtype=torch.float32)
    c.o = torch.as_tensor(rng.integers(0, 60000, size=(c.nb, hkv, BLOCK)), dtype=torch.int32)
    for max_keys, kw in ((16384, dict(keep_first=100, keep_recent=1000)), (20001, {}), (3000, dict(keep_recent=64)),
                         (5, dict(keep_first=5))):
        _plan_case(c, c.w.to(DEV), c.o.to(DEV), max_keys=max_keys, tokens=[60000] * len(S), **kw)


def test_evict_plan_with_unmapped_blocks_and_a_tighter_bound():
    rng = np.random.default_rng(6)
    for seed in range(4):
        c = _plain_cache(np.random.default_rng(seed), [200, 90, 150], 2, unmapped=6)
        _plan_case(c, c.w.to(DEV), c.o.to(DEV), max_keys=40, tokens=None, keep_recent=8)
        _plan_case(c, c.w.to(DEV), c.o.to(DEV), max_keys=100, tokens=None, max_seq_len=160)


def _compact_case(c, source, lens, state=True):
    kc, vc, w, o, bt, _ = c.to(DEV)
    av.verify_kv_compact(kc, vc, bt, _dev(source), _dev(lens), key_weights=w if state else None,
                         key_order=o if state else None)
    torch.cuda.synchronize()
    k, v, rw, ro = bounded.kv_compact(bits(c.k), bits(c.v), bits(c.w), bits(c.o), c.block_tables, source, lens)
    np.testing.assert_array_equal(bits(kc), k)
    np.testing.assert_array_equal(bits(vc), v)
    np.testing.assert_array_equal(bits(w), rw if state else bits(c.w))
    np.testing.assert_array_equal(bits(o), ro if state else bits(c.o))


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("S,hkv,max_keys", [([2], 1, 1), ([100, 33, 0, 64, 65], 2, 40), ([300, 17], 3, 129), ([73], 2, 64),
                                            ([500], 1, 20)])
def test_kv_compact(d, dtype, S, hkv, max_keys):
    rng = np.random.default_rng(d + max_keys)
    c = Cache(rng, S, hkv=hkv, d=d, dtype=dtype, unmapped=1 if len(S) > 2 else 0)
    source, lens = bounded.evict_plan(c.w.numpy(), c.o.numpy(), c.block_tables, c.S, c.nb, max_keys=max_keys)
    _compact_case(c, source, lens)


def test_kv_compact_of_a_plan_with_slots_outside_the_cache():
    rng = np.random.default_rng(1)
    c = Cache(rng, [60, 60], hkv=1, d=64, dtype="bf16")
    source = np.tile(np.arange(32, dtype=np.int32), (2, 1, 1))
    source[0, 0, :4] = [-1, 10 ** 9, 64, 59]
    source[1, 0, 20:24] = [-2 ** 31, 2 ** 31 - 1, 40, 41]
    _compact_case(c, source, [32, 23])
    _compact_case(c, source, [32, 100], state=False)  # a length past the plan
    _compact_case(c, source, [0, -5])


def _attend(q, ks, vs, scale):
    s = np.einsum("hd,td->ht", q, ks) * scale
    p = np.exp(s - s.max(axis=1, keepdims=True))
    return (p / p.sum(axis=1, keepdims=True)) @ vs


def test_a_bounded_session_step_by_step():
    """Prompts, then steps of accepted and rejected drafts on caches that are brought
    back to their bound: at every step the attention sees exactly the kept tokens (by
    their ordinals, from a record of every token's key and value), and the kept ones
    are those the oracle picks."""
    rng = np.random.default_rng(12)
    hkv, G, d, bound, first, recent = 2, 4, 64, 48, 2, 12
    B, nbmax = 3, 12
    nb = B * nbmax + 2
    bt = _dev(rng.permutation(nb)[:B * nbmax].reshape(B, nbmax))
    t16 = torch.bfloat16
    kc = torch.full((nb, hkv, d // 8, 16, 8), float("nan"), dtype=t16, device=DEV)
    # verify_attention multiplies the values behind a request's last key, in the same
    # block, by weights of zero: they may be anything finite, but not NaN
    vc = torch.full((nb, hkv, d, 16), -1e4, dtype=t16, device=DEV)
    w = torch.full((nb, hkv, 16), float("nan"), device=DEV)
    o = torch.full((nb, hkv, 16), -1, dtype=torch.int32, device=DEV)
    freq = torch.as_tensor(10000.0 ** (-np.arange(d // 2) / (d // 2)), device=DEV)
    axes = tuple(f % 3 for f in range(d // 2))
    held = np.zeros(B, dtype=np.int32)   # cached keys
    seen = np.zeros(B, dtype=np.int32)   # tokens so far
    record = [{} for _ in range(B)]      # ordinal -> (key [Hkv, d], value)
    for step in range(7):
        n = np.array([70, 31, 100] if step == 0 else rng.integers(1, 10, size=B))
        if step == 4:
            n[1] = 0  # a request that sits out
        T = int(n.sum())
        qs = q_start_of(n)
        rows = torch.randn((T, hkv * (G + 2), d), device=DEV).to(t16).split([hkv * G, hkv, hkv], dim=1)
        req = np.repeat(np.arange(B), n)
        ordinal = seen[req] + np.arange(T) - qs[req]
        pos = np.stack([ordinal, ordinal // 7, ordinal % 7]).astype(np.int32)
        S, N = held + n, seen + n
        bounds = dict(max_q_len=int(n.max()), max_seq_len=int(S.max()))
        q = av.verify_rotary_append(*rows, _dev(pos), freq, kc, vc, bt, _dev(S), _dev(qs), axes=axes)
        out = av.verify_attention(q, kc, vc, bt, _dev(S), _dev(qs), **bounds)
        k_rot = bounded.rotary(rows[1].double().cpu().numpy(), pos, freq.cpu().numpy(), axes, False)
        for r in range(T):
            record[req[r]][int(ordinal[r])] = (k_rot[r], rows[2][r].double().cpu().numpy())
        # the last row of every request against the tokens that its cache holds
        table, order = bt.cpu().numpy(), o.cpu().numpy()
        qh = q.double().cpu().numpy()
        for i in range(B):
            if n[i] == 0:
                continue
            for g in range(hkv):
                old = [int(order[table[i, t // 16], g, t % 16]) for t in range(held[i])]
                tokens = old + list(range(seen[i], N[i]))
                assert len(set(tokens)) == len(tokens)
                ks = np.stack([record[i][t][0][g] for t in tokens])
                vs = np.stack([record[i][t][1][g] for t in tokens])
                ref = _attend(qh[qs[i + 1] - 1, g * G:(g + 1) * G], ks, vs, d ** -0.5)
                got = out[int(qs[i + 1]) - 1, g * G:(g + 1) * G].double().cpu().numpy()
                off = np.abs(got - ref).max() / np.abs(ref).max()
                assert off <= 2e-2
        # an acceptance, then the weights of the accepted rows
        emitted = n if step == 0 else np.array([rng.integers(1, x + 1) if x else 0 for x in n])
        ow, oo = w.double().cpu().numpy(), o.cpu().numpy()
        av.verify_key_weights(q, kc, w, o, bt, _dev(S), _dev(qs), num_rows=_dev(emitted), num_tokens=_dev(N), **bounds)
        rw, ro, tol = bounded.key_weights(qh, kc.double().cpu().numpy(), ow, oo, table, S, qs, num_rows=emitted,
                                          num_tokens=N)
        gw = w.double().cpu().numpy()
        ok = ~np.isnan(rw)
        np.testing.assert_array_equal(np.isnan(gw), ~ok)
        assert (np.abs(gw - rw)[ok] <= tol[ok]).all()
        np.testing.assert_array_equal(o.cpu().numpy(), ro)
        held, seen = held + emitted, seen + emitted
        src, lens = av.verify_evict_plan(w, o, bt, _dev(held), max_keys=bound, keep_first=first, keep_recent=recent,
                                         max_seq_len=int(held.max()), num_tokens=_dev(seen))
        rs, rl = bounded.evict_plan(gw, ro, table, held, nb, max_keys=bound, keep_first=first, keep_recent=recent,
                                    num_tokens=seen)
        np.testing.assert_array_equal(src.cpu().numpy(), rs)
        av.verify_kv_compact(kc, vc, bt, src, lens, key_weights=w, key_order=o)
        held = lens.cpu().numpy().copy()
        np.testing.assert_array_equal(held, rl)
        for i in range(B):
            for g in range(hkv):
                kept = {int(o[table[i, t // 16], g, t % 16]) for t in range(held[i])}
                assert set(range(min(first, seen[i]))) <= kept
                assert set(range(max(0, seen[i] - recent), seen[i])) <= kept


def test_captured_and_replayed():
    """The four calls in one graph, replayed with eager work between, against the eager
    calls."""
    rng = np.random.default_rng(3)
    S, n = [90, 200, 64], [5, 9, 1]
    c = Cache(rng, S, hkv=2, d=128, dtype="bf16")
    state = c.to(DEV)
    q, k, v = (torch.randn((15, h, 128), device=DEV).to(torch.bfloat16) for h in (8, 2, 2))
    pos = _dev(rng.integers(0, 5000, size=(1, 15)))
    freq = torch.as_tensor(10000.0 ** (-np.arange(64) / 64), device=DEV)
    qs = _dev(q_start_of(n))
    ws = torch.empty(av.key_weights_workspace_size(q, state[0], state[4], max_q_len=9, max_seq_len=200),
                     dtype=torch.uint8, device=DEV)
    pws = torch.empty(av.evict_plan_workspace_size(3, 2, state[4].shape[1], max_seq_len=200, max_keys=60),
                      dtype=torch.uint8, device=DEV)
    qo = torch.empty_like(q)
    src = torch.empty((3, 2, 60), dtype=torch.int32, device=DEV)
    lens = torch.empty((3,), dtype=torch.int32, device=DEV)

    def step():
        kc, vc, w, o, bt, sl = state
        av.verify_rotary_append(q, k, v, pos, freq, kc, vc, bt, sl, qs, q_out=qo)
        av.verify_key_weights(qo, kc, w, o, bt, sl, qs, max_q_len=9, max_seq_len=200, workspace=ws)
        av.verify_evict_plan(w, o, bt, sl, max_keys=60, keep_recent=8, max_seq_len=200, source=src, new_lens=lens,
                             workspace=pws)
        av.verify_kv_compact(kc, vc, bt, src, lens, key_weights=w, key_order=o)

    def reset():
        for x, y in zip(state, c.to(DEV)):
            x.copy_(y)

    step()
    torch.cuda.synchronize()
    want = [bits(x) for x in state[:4]] + [bits(src), bits(lens), bits(qo)]
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        reset()
        ws.random_()
        pws.random_()
        graph.replay()
        torch.cuda.synchronize()
        got = [bits(x) for x in state[:4]] + [bits(src), bits(lens), bits(qo)]
        for a, b in zip(got, want):
            np.testing.assert_array_equal(a, b)


def test_on_another_stream_and_side_by_side():
    """Calls on a stream of their own, whose workspaces and outputs the binding makes,
    with other calls on the current stream at the same time."""
    rng = np.random.default_rng(4)
    S, n = [900, 400], [9, 3]
    c = Cache(rng, S, hkv=2, d=64, dtype="bf16", lost=[50, 60])
    q = torch.randn((12, 8, 64), device=DEV).to(torch.bfloat16)
    qs = _dev(q_start_of(n))
    side = torch.cuda.Stream()

    def calls(stream, outs):
        kc, vc, w, o, bt, sl = c.to(DEV)
        torch.cuda.synchronize()
        av.verify_key_weights(q, kc, w, o, bt, sl, qs, max_q_len=9, max_seq_len=900, num_tokens=_dev(c.tokens),
                              stream=stream)
        src, lens = av.verify_evict_plan(w, o, bt, sl, max_keys=128, max_seq_len=900, num_tokens=_dev(c.tokens),
                                         stream=stream)
        av.verify_kv_compact(kc, vc, bt, src, lens, key_weights=w, key_order=o, stream=stream)
        outs.append((kc, vc, w, o, src))

    outs = []
    calls(None, outs)
    torch.cuda.synchronize()
    for _ in range(4):
        calls(side, outs)
        calls(None, outs)
    torch.cuda.synchronize()
    for other in outs[1:]:
        for a, b in zip(outs[0], other):
            np.testing.assert_array_equal(bits(a), bits(b))


def test_workspace_of_a_larger_batch_serves_smaller_ones():
    """The size asked for one batch covers every batch of fewer requests and rows."""
    def size(B, T, hq, hkv, mq, ms, nb):
        q = torch.empty((T, hq, 128), dtype=torch.bfloat16)
        kc = torch.empty((nb, hkv, 16, 16, 8), dtype=torch.bfloat16)
        bt = torch.empty((B, -(-ms // 16)), dtype=torch.int32)
        return av.key_weights_workspace_size(q, kc, bt, max_q_len=mq, max_seq_len=ms)
    for mq, ms, hq, hkv, nb in ((1, 5000, 8, 8, 1), (1, 5000, 8, 2, 3200), (9, 16384, 32, 8, 1), (200, 4000, 32, 2, 1),
                                (9, 131072, 8, 1, 1)):
        large = size(64, 64 * mq, hq, hkv, mq, ms, nb)
        for B in (1, 2, 3, 7, 20, 63):
            # what the call asks for, not what the query returns
            q = torch.zeros((B * mq, hq, 128), dtype=torch.bfloat16, device=DEV)
            kc = torch.zeros((nb, hkv, 16, 16, 8), dtype=torch.bfloat16, device=DEV)
            bt = torch.zeros((B, -(-ms // 16)), dtype=torch.int32, device=DEV)
            w, o = torch.zeros((nb, hkv, 16), device=DEV), torch.zeros((nb, hkv, 16), dtype=torch.int32, device=DEV)
            ws = torch.empty(large, dtype=torch.uint8, device=DEV)
            # requests without keys: the launch has nothing to do
            av.verify_key_weights(q, kc, w, o, bt, torch.zeros(B, dtype=torch.int32, device=DEV),
                                  torch.zeros(B + 1, dtype=torch.int32, device=DEV), max_q_len=mq, max_seq_len=ms,
                                  workspace=ws)
    torch.cuda.synchronize()


def _least(call, most):
    """The fewest bytes of workspace that `call` takes."""
    low, high = 0, most  # high is taken
    while low < high:
        mid = (low + high) // 2
        try:
            call(mid)
            high = mid
        except av.VerifyError as e:
            assert e.status == av.EWORKSPACE
            low = mid + 1
    return high


@pytest.mark.parametrize("S,n,G,dtype", [
    ([300, 40, 1], [1, 1, 1], 4, "bf16"),      # scores in the workspace
    ([500, 77], [9, 3], 4, "bf16"),
    ([700, 400], [300, 220], 4, "bf16"),       # segments
    ([260, 31], [40, 31], 8, "f32"),
])
def test_key_weights_keep_to_their_workspace(S, n, G, dtype):
    """Nothing is written behind the least size that the call takes, and nothing
    depends on what it held."""
    rng = np.random.default_rng(S[0])
    c = Cache(rng, S, hkv=2, d=128, dtype=dtype)
    q = torch.as_tensor(rng.standard_normal((sum(n), 2 * G, 128))).to(workload.torch_dtype(dtype)).to(DEV)
    kc, _, w0, o0, bt, sl = c.to(DEV)
    kw = dict(max_q_len=max(n), max_seq_len=max(S))
    most = av.key_weights_workspace_size(q, kc, bt, **kw)
    buf = torch.empty(most + 4096, dtype=torch.uint8, device=DEV)
    out = []

    def call(size):
        w, o = w0.clone(), o0.clone()
        av.verify_key_weights(q, kc, w, o, bt, sl, _dev(q_start_of(n)), workspace=buf[:size], **kw)
        out.append((bits(w), bits(o)))

    least = _least(call, most)
    for fill in (0xFF, 0x3C):
        buf.fill_(fill)
        call(least)
        assert (buf[least:] == fill).all()
    for w, o in out[-2:]:
        np.testing.assert_array_equal(w, out[0][0])
        np.testing.assert_array_equal(o, out[0][1])


@pytest.mark.parametrize("S", [[40000, 17000], [200000, 90]])
def test_evict_plan_keeps_to_its_workspace(S):
    rng = np.random.default_rng(7)
    blocks = [-(-s // BLOCK) for s in S]
    bt = torch.full((len(S), max(blocks)), -1, dtype=torch.int32)
    for i, b in enumerate(blocks):
        bt[i, :b] = torch.arange(b) + sum(blocks[:i])
    w = torch.as_tensor(rng.integers(0, 300, size=(sum(blocks), 2, BLOCK)), dtype=torch.float32, device=DEV)
    args = (w, None, bt.to(DEV), _dev(S))
    kw = dict(max_keys=5000, keep_recent=100, max_seq_len=max(S))
    most = av.evict_plan_workspace_size(len(S), 2, max(blocks), max_seq_len=max(S), max_keys=5000)
    buf = torch.empty(most + 4096, dtype=torch.uint8, device=DEV)
    out = []

    def call(size):
        src, lens = av.verify_evict_plan(*args, workspace=buf[:size], **kw)
        out.append((src.cpu().numpy(), lens.cpu().numpy()))

    least = _least(call, most)
    for fill in (0xFF, 0x3C):
        buf.fill_(fill)
        call(least)
        assert (buf[least:] == fill).all()
    rs, rl = bounded.evict_plan(w.double().cpu().numpy(), None, bt.numpy(), S, sum(blocks), max_keys=5000, keep_recent=100)
    for src, lens in out[-2:]:
        np.testing.assert_array_equal(src, rs)
        np.testing.assert_array_equal(lens, rl)
