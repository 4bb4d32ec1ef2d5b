"""verify_norm_rotary and verify_norm_rotary_append against the oracle, and the append
against verify_norm_rotary followed by verify_kv_append, bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
import workload
from bounded_common import Cache, bits, q_start_of
from oracle import serving

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6

CASES = [
    # T, Hq, Hkv, D, dtype, rot, axes, interleaved, scale
    (1, 8, 2, 128, "bf16", 128, 1, False, 0.0),
    (17, 5, 1, 64, "bf16", 64, 3, False, 1.25),
    (100, 8, 8, 128, "bf16", 64, 2, True, 0.0),
    (50, 6, 2, 128, "bf16", 96, 1, False, 0.0),   # ten items of 16
    (33, 4, 2, 128, "bf16", 38, 4, False, 0.5),   # frequencies that fill no 16 bytes
    (16, 6, 3, 64, "bf16", 6, 1, True, 0.0),
    (15, 8, 2, 64, "f32", 64, 3, True, 0.0),
    (40, 3, 1, 128, "f32", 128, 2, False, 2.0),
    (21, 3, 2, 128, "f32", 64, 1, True, 0.0),     # all 32 lanes
    (47, 4, 4, 128, "f32", 2, 1, False, 0.0),
    (700, 40, 8, 128, "bf16", 128, 3, False, 0.0),
]


def _freqs(F):
    return 10000.0 ** (-np.arange(F) / F)


def _inputs(rng, T, Hq, Hkv, D, dtype, rot, A):
    F = rot // 2
    axes = [f % A for f in range(F)]
    dt = workload.torch_dtype(dtype)
    # heads of very different lengths, one of zeros
    size = np.exp(2 * rng.standard_normal((T, Hq + 2 * Hkv, 1)))
    x = rng.standard_normal((T, Hq + 2 * Hkv, D)) * size
    x[T // 2, 0] = 0
    x = torch.as_tensor(x).to(dt)
    pos = rng.integers(-5, 200000, size=(A, T)).astype(np.int32)
    w = [torch.as_tensor(1 + 0.3 * rng.standard_normal(D), dtype=torch.float32) for _ in range(2)]
    return x, pos, axes, _freqs(F), w


def _close(got, x, weight, pos, freq, axes, interleaved, scale, dtype):
    """Half a step of the storage type.  The norm: a sum of squares by chains of at most
    16 and six exchanges, mean and eps (24 half steps, halved by the root), the root's two,
    two products: 16 of 2^-24.  The rotation: seven (products, sum, factor, sine and
    cosine), and the angle's own error."""
    y = serving.head_norm(x, weight, EPS)
    ref = serving.norm_rotary(x, weight, EPS, pos, freq, axes, interleaved, scale)
    F = len(axes)
    tol = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype] * np.abs(ref)
    tol[:, :, 2 * F:] += 16 * 2.0 ** -24 * np.abs(y[:, :, 2 * F:]) * (1 + 2.0 ** -7)
    angle = np.abs(np.asarray(pos, dtype=np.float64)[list(axes)].T * freq)
    off = (23 * 2.0 ** -24 + np.pi * 2.0 ** -24 + 3 * 2.0 ** -53 * angle)[:, None, :]
    for f in range(F):
        a, b = (2 * f, 2 * f + 1) if interleaved else (f, f + F)
        size = scale * (np.abs(y[:, :, a]) + np.abs(y[:, :, b])) * off[:, :, f] * (1 + 2.0 ** -7)
        tol[:, :, a] += size
        tol[:, :, b] += size
    got = got.to(torch.float64).cpu().numpy()
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), "%d of %d off, worst %.3g of its tolerance" % (
        bad.sum(), bad.size, (np.abs(got - ref) / np.maximum(tol, 1e-300)).max())


@pytest.mark.parametrize("T,Hq,Hkv,D,dtype,rot,A,inter,scale", CASES)
def test_norm_rotary(T, Hq, Hkv, D, dtype, rot, A, inter, scale):
    rng = np.random.default_rng(T + rot)
    x, pos, axes, freq, w = _inputs(rng, T, Hq, Hkv, D, dtype, rot, A)
    dev = x.to(DEV)
    q, k = dev[:, :Hq], dev[:, Hq:Hq + Hkv]  # slices of wider rows
    args = dict(q_weight=w[0].to(DEV), k_weight=w[1].to(DEV), eps=EPS, axes=axes, interleaved=inter, scale=scale)
    p, f = torch.as_tensor(pos, device=DEV), torch.as_tensor(freq, device=DEV)
    qo, ko = av.verify_norm_rotary(q, k, p, f, **args)
    x64 = x.to(torch.float64).numpy()
    s = scale or 1.0
    _close(qo, x64[:, :Hq], w[0].double().numpy(), pos, freq, axes, inter, s, dtype)
    _close(ko, x64[:, Hq:Hq + Hkv], w[1].double().numpy(), pos, freq, axes, inter, s, dtype)
    np.testing.assert_array_equal(bits(dev), bits(x))
    # contiguous, in place, without keys and on another stream: the same bits (weights of
    # one and no weights too)
    qc, kc = q.contiguous(), k.contiguous()
    assert av.verify_norm_rotary(qc, kc, p, f, q_out=qc, k_out=kc, **args)[0] is qc
    np.testing.assert_array_equal(bits(qc), bits(qo))
    np.testing.assert_array_equal(bits(kc), bits(ko))
    args.update(q_weight=None, k_weight=torch.ones(D, device=DEV))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q1, none = av.verify_norm_rotary(q, None, p, f, stream=side, **args)
    side.synchronize()
    args.update(q_weight=torch.ones(D, device=DEV))
    q2, _ = av.verify_norm_rotary(q, None, p, f, **args)
    assert none is None
    np.testing.assert_array_equal(bits(q1), bits(q2))


@pytest.mark.parametrize("dtype,D,rot,inter", [("bf16", 128, 128, False), ("bf16", 64, 32, True), ("f32", 64, 64, False),
                                                ("bf16", 128, 38, False)])
@pytest.mark.parametrize("S,n,unmapped", [
    ([1], [1], 0),
    ([33, 16, 5, 100], [9, 16, 0, 3], 0),
    ([300, 41], [300, 41], 1),                    # prompts, one with an unmapped block
    (list(range(20, 60)), [1 + i % 4 for i in range(40)], 0),
])
def test_append(dtype, D, rot, inter, S, n, unmapped):
    Hq, Hkv, A = 6, 3, 2
    rng = np.random.default_rng(sum(S))
    cache = Cache(rng, S, hkv=Hkv, d=D, dtype=dtype, unmapped=unmapped)
    T = sum(n) + 2  # two rows behind the last request's: rotated, not stored
    x, pos, axes, freq, w = _inputs(rng, T, Hq, Hkv, D, dtype, rot, A)
    dev = x.to(DEV)
    q, k, v = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:]
    args = dict(q_weight=w[0].to(DEV), k_weight=w[1].to(DEV), eps=EPS, axes=axes, interleaved=inter)
    p, f = torch.as_tensor(pos, device=DEV), torch.as_tensor(freq, device=DEV)
    kc, vc, _, _, bt, sl = cache.to(DEV)
    qs = torch.as_tensor(q_start_of(n), device=DEV)
    qo = av.verify_norm_rotary_append(q, k, v, p, f, kc, vc, bt, sl, qs, **args)
    q1, k1 = av.verify_norm_rotary(q, k, p, f, **args)
    kc1, vc1, _, _, _, _ = cache.to(DEV)
    last = sum(n)
    av.verify_kv_append(k1[:last].contiguous(), v[:last].contiguous(), kc1, vc1, bt, sl, qs)
    for a, b in ((qo, q1), (kc, kc1), (vc, vc1)):
        np.testing.assert_array_equal(bits(a), bits(b))


def test_a_captured_call_is_replayed_on_new_rows():
    rng = np.random.default_rng(5)
    x, pos, axes, freq, w = _inputs(rng, 24, 4, 2, 64, "bf16", 64, 1)
    dev, p, f = x.to(DEV), torch.as_tensor(pos, device=DEV), torch.as_tensor(freq, device=DEV)
    q, k = dev[:, :4].contiguous(), dev[:, 4:6].contiguous()
    args = dict(q_weight=w[0].to(DEV), eps=EPS, axes=axes)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    av.verify_norm_rotary(q, k, p, f, q_out=qo, k_out=ko, **args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        av.verify_norm_rotary(q, k, p, f, q_out=qo, k_out=ko, **args)
    for step in range(3):
        q.mul_(-1.5)
        p.add_(7)
        g.replay()
        torch.cuda.synchronize()
        got = bits(qo)
        want, _ = av.verify_norm_rotary(q, k, p, f, **args)
        np.testing.assert_array_equal(got, bits(want))


def test_heads_that_are_not_finite_stay_apart():
    q = torch.randn((5, 4, 128), device=DEV, dtype=torch.bfloat16)
    want, _ = av.verify_norm_rotary(q, None, torch.arange(5, dtype=torch.int32, device=DEV),
                                    torch.as_tensor(_freqs(64), device=DEV))
    q[2, 1, 7] = float("nan")
    q[3, 0, 5] = float("inf")
    got, _ = av.verify_norm_rotary(q, None, torch.arange(5, dtype=torch.int32, device=DEV),
                                   torch.as_tensor(_freqs(64), device=DEV))
    assert got[2, 1].isnan().all() and got[3, 0, 5].isnan()
    mine = torch.ones((5, 4), dtype=torch.bool, device=DEV)
    mine[2, 1] = mine[3, 0] = False
    np.testing.assert_array_equal(bits(got[mine]), bits(want[mine]))
