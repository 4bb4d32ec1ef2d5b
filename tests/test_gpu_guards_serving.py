"""Buffer guards (see test_gpu_guards) of the norms with the rotation, the shared
attention, the changed logits and the token counts."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
from bounded_common import Cache, q_start_of
from oracle import serving
from shared_common import SharedBatch
from test_gpu_guards import Arena, _assert_unchanged, _bytes, _snapshot, _twice, say

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = torch.int32


def _dev(x, dtype=None):
    return torch.as_tensor(x, dtype=dtype).to(DEV)


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 8, 2, 128), ("bf16", 8, 1, 64), ("f32", 6, 3, 128)])
@pytest.mark.parametrize("wide", [False, True], ids=["", "wide"])
@pytest.mark.parametrize("name,groups,S,n", [
    ("tall", [(6, 400)], [420 + 31 * i for i in range(6)], [9] * 6),
    ("flat", [(2, 1000), (0, 30), (1, 64)], [1001, 1010, 70, 33], [1, 2, 1, 1]),
    ("prompts", [(2, 96)], [400, 96], [300, 50]),
    ("many", [(200, 32), (90, 48)], [49 + i % 31 for i in range(300)], [1 + i % 3 for i in range(300)]),
])
def test_shared_attention(name, groups, S, n, dtype, hq, hkv, d, wide):
    b = SharedBatch(11, groups, S, n, hq=hq, hkv=hkv, d=d, dtype=dtype, sinks=True, wide=wide)
    args = b.to(DEV)
    sinks = b.sinks.to(DEV)
    size = av.attention_shared_workspace_size(args[0], args[1], args[3], num_groups=len(groups), **b.bounds)
    arena = Arena()
    out = arena.take("out", tuple(args[0].shape), args[0].dtype)
    ws = arena.take("workspace", (size,), torch.uint8)
    _twice(lambda: av.verify_attention_shared(*args, sinks=sinks, out=out, workspace=ws, **b.bounds), arena,
           args + [sinks], {"out": (out, out.numel())}, "shared attention %s %s" % (name, dtype))


@pytest.mark.parametrize("dtype,D,rot,inter", [("bf16", 128, 128, False), ("bf16", 64, 64, True), ("f32", 128, 128, True),
                                               ("bf16", 128, 38, False)])
def test_norm_rotary(dtype, D, rot, inter):
    rng = np.random.default_rng(4)
    S, n = [33, 16, 70], [9, 1, 20]
    T, Hq, Hkv = sum(n), 6, 2
    cache = Cache(rng, S, hkv=Hkv, d=D, dtype=dtype)
    q, k, v = (torch.randn((T, h, D), device=DEV).to(cache.dtype) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, 90000, (T,), dtype=I32, device=DEV)
    freq = _dev(10000.0 ** (-np.arange(rot // 2) / (rot // 2)))
    w = [torch.rand((D,), device=DEV) + 0.5 for _ in range(2)]
    kw = dict(q_weight=w[0], k_weight=w[1], interleaved=inter)
    arena = Arena()
    qo, ko = arena.take("q_out", tuple(q.shape), q.dtype), arena.take("k_out", tuple(k.shape), k.dtype)
    _twice(lambda: av.verify_norm_rotary(q, k, pos, freq, q_out=qo, k_out=ko, **kw), arena, [q, k, pos, freq, *w],
           {"q_out": (qo, qo.numel()), "k_out": (ko, ko.numel())}, "norm rotary %s %d" % (dtype, rot))
    # the append: what it does not store stays
    kc0, vc0, _, _, bt, sl = cache.to(DEV)
    qs = _dev(q_start_of(n))
    arena = Arena()
    kc, vc = arena.take("k_cache", tuple(kc0.shape), kc0.dtype), arena.take("v_cache", tuple(vc0.shape), vc0.dtype)
    q1 = arena.take("q_out", tuple(q.shape), q.dtype)
    inputs = [q, k, v, pos, freq, *w, bt, sl, qs]
    before = _snapshot(inputs)
    results = []
    for byte in (0xA5, 0x5A):
        arena.fill(byte)
        kc.copy_(kc0)
        vc.copy_(vc0)
        av.verify_norm_rotary_append(q, k, v, pos, freq, kc, vc, bt, sl, qs, q_out=q1, **kw)
        arena.check("norm rotary append")
        results.append([_bytes(t).clone() for t in (kc, vc, q1)])
    _assert_unchanged(inputs, before, "norm rotary append")
    for a, b in zip(*results):
        assert torch.equal(a, b)
    new = torch.zeros(kc.shape, dtype=torch.bool, device=DEV)
    for i in range(len(S)):
        for p in range(S[i] - n[i], S[i]):
            new[int(bt[i, p // 16]), :, :, p % 16] = True
    assert torch.equal(_bytes(kc[~new]), _bytes(kc0[~new]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [5, 2048, 5001])
def test_changed_logits_and_counts(V, dtype):
    rng = np.random.default_rng(V)
    n = [3, 0, 9]
    T, B, slots_n = sum(n), 3, 4
    counts0 = _dev(rng.integers(0, 3, size=(slots_n, V)), I32)
    seen0 = torch.stack([_dev(serving.words(rng.random((slots_n, V)) < 0.2)),
                         _dev(serving.words(counts0.cpu().numpy() > 0))], dim=1).contiguous()
    logits = torch.randn((T, V), device=DEV).to(dtype)
    tokens = _dev(rng.integers(0, V, size=T), I32)
    qs, slots = _dev(q_start_of(n)), _dev([2, 0, 3], I32)
    par = [torch.rand(B, device=DEV) + 0.5 for _ in range(3)]
    mask, rows = _dev(serving.words(rng.random((2, V)) < 0.6)), _dev(rng.integers(-1, 2, size=T), I32)
    bs, bt, bv = _dev([0, 2, 2, 5], I32), _dev(rng.integers(0, V, size=5), I32), torch.randn(5, device=DEV)
    arena = Arena()
    out = arena.take("out", (T, V), dtype)
    call = lambda o: av.verify_adjust_logits(logits, tokens, qs, counts=counts0, seen=seen0, slots=slots, repetition=par[0],
                                             frequency=par[1], presence=par[2], bias_start=bs, bias_tokens=bt,
                                             bias_values=bv, mask=mask, mask_rows=rows, out=o)
    _twice(lambda: call(out), arena, [logits, tokens, qs, slots, *par, mask, rows, bs, bt, bv, counts0, seen0],
           {"out": (out, T * V)}, "changed logits %d" % V)
    # in place
    arena = Arena()
    mine = arena.take("logits", (T, V), dtype)
    mine.copy_(logits)
    want = out.clone()
    given, logits = logits, mine
    call(mine)
    arena.check("changed logits in place %d" % V)
    assert torch.equal(_bytes(mine), _bytes(want))
    # counts
    arena = Arena()
    counts, seen = arena.take("counts", (slots_n, V), I32), arena.take("seen", tuple(seen0.shape), I32)
    emitted = _dev(rng.integers(-1, V + 1, size=T), I32)
    for prompt, many in ((False, 1), (True, 1), (True, 100)):
        tok, start = emitted.repeat(many), qs * many
        inputs = [tok, start, slots]
        before = _snapshot(inputs)
        counts.copy_(counts0)
        seen.copy_(seen0)
        av.verify_count_tokens(counts, seen, tok, start, slots=slots, prompt=prompt)
        arena.check("counts %d" % V)
        _assert_unchanged(inputs, before, "counts")
        c, s = serving.count_tokens(counts0.cpu().numpy(), seen0.cpu().numpy(), tok.cpu().numpy(), start.cpu().numpy(),
                                    slots=[2, 0, 3], prompt=prompt)
        np.testing.assert_array_equal(counts.cpu().numpy(), c)
        np.testing.assert_array_equal(seen.cpu().numpy(), s)
    say("   counts ok")
