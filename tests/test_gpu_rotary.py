"""verify_rotary and verify_rotary_append against the oracle, and the append against
verify_rotary followed by verify_kv_append, bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
import workload
from bounded_common import Cache, bits, q_start_of
from oracle import bounded

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _freqs(F):
    return 10000.0 ** (-np.arange(F) / F)


def _close(got, x, pos, freq, axes, interleaved, scale, dtype):
    """Half a step of the storage type; the rotation's products, sum and factor in fp32
    (three half steps of the pair's size), its sine and cosine (four of 2^-24, and the
    angle's own: its fraction of a turn is rounded to 2^-24 half turns, after three
    roundings of 2^-53 of the whole angle)."""
    ref = bounded.rotary(x, pos, freq, axes, interleaved, scale)
    F = len(axes)
    tol = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype] * np.abs(ref)
    angle = np.abs(np.asarray(pos, dtype=np.float64)[list(axes)].T * freq)
    off = (7 * 2.0 ** -24 + np.pi * 2.0 ** -24 + 3 * 2.0 ** -53 * angle)[:, None, :]
    for f in range(F):
        a, b = (2 * f, 2 * f + 1) if interleaved else (f, f + F)
        size = scale * (np.abs(x[:, :, a]) + np.abs(x[:, :, b])) * off[:, :, f] * (1 + 2.0 ** -7)
        tol[:, :, a] += size
        tol[:, :, b] += size
    got = got.to(torch.float64).cpu().numpy()
    bad = np.abs(got - ref) > tol
    assert not bad.any(), "%d of %d off, worst %.3g of its tolerance" % (
        bad.sum(), bad.size, (np.abs(got - ref) / np.maximum(tol, 1e-300)).max())
    np.testing.assert_array_equal(got[:, :, 2 * F:], x[:, :, 2 * F:])


CASES = [
    # T, Hq, Hkv, D, dtype, rot, axes, interleaved, scale
    (1, 8, 2, 128, "bf16", 128, 1, False, 0.0),
    (17, 5, 1, 64, "bf16", 64, 3, False, 1.25),
    (100, 8, 8, 128, "bf16", 64, 2, True, 0.0),
    (33, 4, 2, 128, "bf16", 38, 4, False, 0.5),   # frequencies that fill no 16 bytes
    (16, 6, 3, 64, "bf16", 6, 1, True, 0.0),
    (15, 8, 2, 64, "f32", 64, 3, True, 0.0),
    (40, 3, 1, 128, "f32", 128, 2, False, 2.0),
    (47, 4, 4, 128, "f32", 2, 1, False, 0.0),
    (700, 40, 8, 128, "bf16", 128, 3, False, 0.0),  # several workgroups per tile and many tiles
]


def _inputs(rng, T, Hq, Hkv, D, dtype, rot, A):
    F = rot // 2
    axes = [f % A for f in range(F)]
    pos = rng.integers(-5, 300000, size=(A, T)).astype(np.int32)
    pos[0, 0] = 2 ** 31 - 1
    pos[-1, T // 2] = -2 ** 31
    t = workload.torch_dtype(dtype)
    x = [torch.as_tensor(rng.standard_normal((T, h, D))).to(t) for h in (Hq, Hkv, Hkv)]
    return axes, pos, _freqs(F), x


@pytest.mark.parametrize("T,Hq,Hkv,D,dtype,rot,A,interleaved,scale", CASES)
@pytest.mark.parametrize("layout", ["plain", "fused", "odd"])
def test_rotary(T, Hq, Hkv, D, dtype, rot, A, interleaved, scale, layout):
    rng = np.random.default_rng(T + rot)
    axes, pos, freq, (q, k, v) = _inputs(rng, T, Hq, Hkv, D, dtype, rot, A)
    dq, dk = q.to(DEV), k.to(DEV)
    if layout == "fused":  # slices of one projection's rows
        dq, dk, _ = torch.cat([q, k, v], dim=1).to(DEV).split([Hq, Hkv, Hkv], dim=1)
    elif layout == "odd":  # one element off any alignment
        def odd(x):
            buf = torch.empty(x.numel() + 1, dtype=x.dtype, device=DEV)
            buf[1:] = x.to(DEV).reshape(-1)
            return buf[1:].view(x.shape)
        dq, dk = odd(q), odd(k)
    kw = dict(axes=axes, interleaved=interleaved, scale=scale)
    dpos, dfreq = torch.as_tensor(pos, device=DEV), torch.as_tensor(freq, device=DEV)
    q_out, k_out = av.verify_rotary(dq, dk, dpos, dfreq, **kw)
    torch.cuda.synchronize()
    for got, x in ((q_out, q), (k_out, k)):
        _close(got, x.double().numpy(), pos, freq, axes, interleaved, scale or 1.0, dtype)
    # the inputs are as they were, and in place gives the same bits
    np.testing.assert_array_equal(bits(dq), bits(q))
    av.verify_rotary(dq, dk, dpos, dfreq, q_out=dq, k_out=dk, **kw)
    np.testing.assert_array_equal(bits(dq), bits(q_out))
    np.testing.assert_array_equal(bits(dk), bits(k_out))
    alone, none = av.verify_rotary(q.to(DEV), None, dpos, dfreq, **kw)
    assert none is None
    np.testing.assert_array_equal(bits(alone), bits(q_out))


def test_rotary_keeps_values_that_are_not_finite_to_their_pairs():
    q = torch.ones((2, 1, 64), dtype=torch.bfloat16, device=DEV)
    q[0, 0, 3] = float("nan")
    q[1, 0, 40] = float("inf")
    out, _ = av.verify_rotary(q, None, torch.tensor([7, 9], dtype=torch.int32, device=DEV),
                              torch.as_tensor(_freqs(16), device=DEV))
    bad = ~torch.isfinite(out[:, 0].float().cpu())
    assert bad.nonzero().tolist() == [[0, 3], [0, 19], [1, 40]]


def _append_case(rng, S, n, Hq, Hkv, D, dtype, rot, A, unmapped=0):
    c = Cache(rng, S, hkv=Hkv, d=D, dtype=dtype, unmapped=unmapped)
    T = int(np.sum(n))
    axes, pos, freq, x = _inputs(rng, T, Hq, Hkv, D, dtype, rot, A)
    return c, q_start_of(n), axes, pos, freq, x


@pytest.mark.parametrize("S,n,Hq,Hkv,D,dtype,rot,A,interleaved,unmapped", [
    ([9], [1], 8, 2, 128, "bf16", 128, 1, False, 0),
    ([300, 0, 40, 16, 1], [9, 0, 40, 5, 1], 8, 2, 128, "bf16", 128, 3, False, 0),
    ([70, 31, 200], [70, 31, 33], 8, 4, 64, "bf16", 32, 2, True, 2),
    ([70, 31, 200], [33, 7, 2], 6, 3, 64, "bf16", 38, 2, False, 1),
    ([50, 90, 17], [17, 3, 17], 4, 1, 128, "f32", 128, 4, True, 0),
    ([50, 90, 17], [1, 50, 16], 4, 2, 64, "f32", 64, 1, False, 2),
])
@pytest.mark.parametrize("fused", [False, True])
def test_rotary_append(S, n, Hq, Hkv, D, dtype, rot, A, interleaved, unmapped, fused):
    rng = np.random.default_rng(len(S) + D)
    c, qs, axes, pos, freq, (q, k, v) = _append_case(rng, S, n, Hq, Hkv, D, dtype, rot, A, unmapped)
    rows = [q.to(DEV), k.to(DEV), v.to(DEV)]
    if fused:
        rows = torch.cat([q, k, v], dim=1).to(DEV).split([Hq, Hkv, Hkv], dim=1)
    kc, vc, _, _, bt, sl = c.to(DEV)
    dqs = torch.as_tensor(qs, device=DEV)
    kw = dict(axes=axes, interleaved=interleaved)
    dpos, dfreq = torch.as_tensor(pos, device=DEV), torch.as_tensor(freq, device=DEV)
    q_out = av.verify_rotary_append(*rows, dpos, dfreq, kc, vc, bt, sl, dqs, **kw)
    torch.cuda.synchronize()
    _close(q_out, q.double().numpy(), pos, freq, axes, interleaved, 1.0, dtype)
    kc2, vc2, _, _, _, _ = c.to(DEV)
    q2, k2 = av.verify_rotary(*rows[:2], dpos, dfreq, **kw)
    av.verify_kv_append(k2, v.to(DEV), kc2, vc2, bt, sl, dqs)
    for a, b in ((q_out, q2), (kc, kc2), (vc, vc2)):
        np.testing.assert_array_equal(bits(a), bits(b))
    # and something was written: the last token of the first request
    b = c.block_tables[0, (S[0] - 1) // 16]
    if 0 <= b < c.nb:
        np.testing.assert_array_equal(bits(vc[int(b), :, :, (S[0] - 1) % 16]), bits(v[qs[1] - 1]))


def test_rotary_append_of_rows_in_front_of_the_cache_and_of_no_request():
    """A request with more rows than keys (its first rows have no slot), and rows past
    the last request: rotated, not stored."""
    rng = np.random.default_rng(5)
    c, qs, axes, pos, freq, (q, k, v) = _append_case(rng, [3, 20], [3, 20], 4, 2, 64, "bf16", 64, 1)
    qs = np.array([0, 8, 20], dtype=np.int32)  # 8 rows of a 3-key request; rows 20 .. 22 of none
    kc, vc, _, _, bt, sl = c.to(DEV)
    args = [torch.as_tensor(x, device=DEV) for x in (pos, freq)]
    q_out = av.verify_rotary_append(q.to(DEV), k.to(DEV), v.to(DEV), *args, kc, vc, bt, sl,
                                    torch.as_tensor(qs, device=DEV))
    _close(q_out, q.double().numpy(), pos, freq, axes, False, 1.0, "bf16")
    kc2, vc2, _, _, _, _ = c.to(DEV)
    _, k2 = av.verify_rotary(q.to(DEV), k.to(DEV), *args)
    av.verify_kv_append(k2, v.to(DEV), kc2, vc2, bt, sl, torch.as_tensor(qs, device=DEV))
    np.testing.assert_array_equal(bits(kc), bits(kc2))
    np.testing.assert_array_equal(bits(vc), bits(vc2))


@pytest.mark.parametrize("B", [1023, 1024, 1025, 5000])
def test_rotary_append_of_many_requests(B):
    """More requests than the search keeps in LDS, empty ones among them."""
    rng = np.random.default_rng(B)
    n = rng.integers(0, 3, size=B)
    n[rng.integers(0, B, size=B // 2)] = 0
    c, qs, axes, pos, freq, (q, k, v) = _append_case(rng, n + rng.integers(0, 4, size=B), n, 2, 1, 64, "bf16", 64, 1)
    kc, vc, _, _, bt, sl = c.to(DEV)
    kc2, vc2, _, _, _, _ = c.to(DEV)
    args = [torch.as_tensor(x, device=DEV) for x in (pos, freq)]
    dqs = torch.as_tensor(qs, device=DEV)
    av.verify_rotary_append(q.to(DEV), k.to(DEV), v.to(DEV), *args, kc, vc, bt, sl, dqs)
    _, k2 = av.verify_rotary(q.to(DEV), k.to(DEV), *args)
    av.verify_kv_append(k2, v.to(DEV), kc2, vc2, bt, sl, dqs)
    np.testing.assert_array_equal(bits(kc), bits(kc2))
    np.testing.assert_array_equal(bits(vc), bits(vc2))


def test_rotary_of_no_rows_and_no_requests():
    e = lambda *s: torch.empty(s, dtype=torch.bfloat16, device=DEV)
    pos = torch.empty((1, 0), dtype=torch.int32, device=DEV)
    freq = torch.as_tensor(_freqs(32), device=DEV)
    q, k = av.verify_rotary(e(0, 4, 64), e(0, 2, 64), pos, freq)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    # rows that belong to no request: the queries are rotated all the same
    q = torch.randn((3, 4, 64), device=DEV).to(torch.bfloat16)
    pos = torch.tensor([[4, 5, 6]], dtype=torch.int32, device=DEV)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    out = av.verify_rotary_append(q, e(3, 2, 64), e(3, 2, 64), pos, freq, e(1, 2, 8, 16, 8), e(1, 2, 64, 16),
                                  i32(0, 1), i32(0), i32(1))
    np.testing.assert_array_equal(bits(out), bits(av.verify_rotary(q, None, pos, freq)[0]))
