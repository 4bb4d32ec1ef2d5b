"""Norms with the rotation, changed logits and token counts on the host: every refusal
comes before the GPU is touched, from the library and from the binding."""
from __future__ import annotations

import ctypes

import pytest
import torch

import paper_2608_24004_amd as av
from test_abi_bounded_cpu import DUMMY, _attn, _rot


def _norm(p, T=3, hq=8, hkv=2, q=DUMMY, qs=1024, k=DUMMY, ks=256, qw=DUMMY, kw=None, eps=1e-6, pos=DUMMY, freq=DUMMY,
          qo=DUMMY, qos=1024, ko=DUMMY, kos=256):
    return av.library().verify_norm_rotary(ctypes.byref(p) if p is not None else None, T, hq, hkv, q, qs, k, ks, qw, kw,
                                           eps, pos, freq, qo, qos, ko, kos, None)


def _norm_append(attn=None, p=None, T=3, eps=1e-6, kc=DUMMY, v=DUMMY, qos=1024, bt=DUMMY):
    return av.library().verify_norm_rotary_append(
        ctypes.byref(attn or _attn()), ctypes.byref(p or _rot()), T, DUMMY, 1024, DUMMY, 256, v, 256, None, DUMMY, eps,
        DUMMY, DUMMY, bt, DUMMY, DUMMY, DUMMY, qos, kc, DUMMY, None)


@pytest.mark.parametrize("kw,want", [
    (dict(eps=-1.0), av.EINVAL), (dict(eps=float("nan")), av.EINVAL), (dict(eps=float("inf")), av.EINVAL),
    (dict(T=-1), av.EINVAL), (dict(hq=0), av.EINVAL), (dict(q=None), av.EINVAL), (dict(pos=None), av.EINVAL),
    (dict(k=None), av.EINVAL), (dict(ko=None), av.EINVAL), (dict(qs=1023), av.EINVAL), (dict(kos=255), av.EINVAL),
    (dict(qs=2048), av.EINVAL), (dict(hq=40000, qs=1 << 40, qos=1 << 40), av.EUNSUPPORTED),
    (dict(T=2 ** 31 - 1), av.EUNSUPPORTED), (dict(T=0, q=None), av.OK),
])
def test_norm_rotary(kw, want):
    assert _norm(_rot(), **kw) == want
    assert _norm(None) == av.EINVAL and _norm(_rot(head_dim=96)) == av.EUNSUPPORTED


@pytest.mark.parametrize("kw,want", [
    (dict(eps=-1.0), av.EINVAL), (dict(kc=ctypes.c_void_p(0x1008)), av.EINVAL), (dict(v=None), av.EINVAL),
    (dict(bt=None), av.EINVAL), (dict(qos=1000), av.EINVAL), (dict(qos=2048), av.EINVAL),
    (dict(p=_rot(dtype=av.F32)), av.EINVAL), (dict(attn=_attn(head_dim=64)), av.EINVAL),
    (dict(attn=_attn(block_size=32)), av.EUNSUPPORTED), (dict(T=0), av.OK),
])
def test_norm_rotary_append(kw, want):
    assert _norm_append(**kw) == want


def _adjust(B=2, T=5, V=100, rs=0, dtype=av.BF16, logits=DUMMY, tokens=DUMMY, qs=DUMMY, out=ctypes.c_void_p(0x9000), os=0,
            params=True, **kw):
    p = av.AdjustParams()
    for k, v in kw.items():
        setattr(p, k, v)
    return av.library().verify_adjust_logits(B, T, V, rs, dtype, logits, tokens, qs, ctypes.byref(p) if params else None,
                                             out, os, None)


@pytest.mark.parametrize("kw,want", [
    (dict(params=False), av.EINVAL), (dict(B=-1), av.EINVAL), (dict(T=-1), av.EINVAL), (dict(V=0), av.EINVAL),
    (dict(V=2 ** 31 - 2049), av.EUNSUPPORTED), (dict(V=2 ** 33), av.EUNSUPPORTED), (dict(dtype=2), av.EUNSUPPORTED),
    (dict(B=65536), av.EUNSUPPORTED), (dict(rs=99), av.EINVAL), (dict(os=-1), av.EINVAL),
    (dict(logits=None), av.EINVAL), (dict(qs=None), av.EINVAL), (dict(out=None), av.EINVAL),
    (dict(out=DUMMY, rs=128), av.EINVAL),                       # in place with two strides
    (dict(repetition=0x1000), av.EINVAL),                       # no state
    (dict(frequency=0x1000, counts=0x1000), av.EINVAL),
    (dict(presence=0x1000, counts=0x1000, seen=0x1000, tokens=None), av.EINVAL),
    (dict(presence=0x1000, counts=0x1000, seen=0x1000, num_slots=-1), av.EINVAL),
    (dict(bias_start=0x1000, num_biases=1), av.EINVAL), (dict(bias_start=0x1000, num_biases=-1), av.EINVAL),
    (dict(mask_rows=0x1000, num_masks=1), av.EINVAL), (dict(mask_rows=0x1000, num_masks=-1), av.EINVAL),
    (dict(T=0, logits=None), av.OK), (dict(B=0, qs=None), av.OK),
])
def test_adjust_logits(kw, want):
    assert _adjust(**kw) == want


def test_adjust_logits_refuses_more_rows_than_its_parts_count():
    assert _adjust(T=2 ** 30) == av.EUNSUPPORTED and _adjust(T=2 ** 31 - 1) == av.EUNSUPPORTED
    assert _adjust(T=2 ** 30 - 1, out=None) == av.EINVAL


def _count(B=2, total=5, V=100, slots_n=3, tokens=DUMMY, start=DUMMY, prompt=0, counts=DUMMY, seen=DUMMY):
    return av.library().verify_count_tokens(B, total, V, slots_n, tokens, start, None, None, prompt, counts, seen, None)


@pytest.mark.parametrize("kw,want", [
    (dict(B=-1), av.EINVAL), (dict(total=-1), av.EINVAL), (dict(V=0), av.EINVAL), (dict(slots_n=-1), av.EINVAL),
    (dict(prompt=2), av.EINVAL), (dict(V=2 ** 31), av.EUNSUPPORTED), (dict(B=65536), av.EUNSUPPORTED),
    (dict(tokens=None), av.EINVAL), (dict(start=None), av.EINVAL), (dict(seen=None), av.EINVAL),
    (dict(counts=None), av.EINVAL), (dict(B=0), av.OK), (dict(total=0, counts=None), av.OK), (dict(slots_n=0), av.OK),
])
def test_count_tokens(kw, want):
    assert _count(**kw) == want


def _shared(attn=None, T=5, mq=3, ms=5000, G=1, mp=64, q=DUMMY, kc=DUMMY, vc=DUMMY, gs=DUMMY, pl=DUMMY, out=DUMMY, ws=DUMMY,
            size=None):
    params = attn or _attn(max_blocks_per_seq=400)
    if size is None:
        n = ctypes.c_size_t(0)
        rc = av.library().verify_attention_shared_workspace_size(ctypes.byref(params), T, mq, ms, G, mp, ctypes.byref(n))
        size = n.value if rc == av.OK else 0
    return av.library().verify_attention_shared(ctypes.byref(params), T, mq, ms, G, mp, q, kc, vc, DUMMY, DUMMY, DUMMY, gs,
                                                pl, None, out, ws, size, None)


@pytest.mark.parametrize("kw,want", [
    (dict(attn=_attn(sliding_window=5)), av.EUNSUPPORTED), (dict(attn=_attn(kv_split_blocks=1)), av.EUNSUPPORTED),
    (dict(attn=_attn(head_dim=96)), av.EUNSUPPORTED), (dict(attn=_attn(num_q_heads=7)), av.EINVAL),
    (dict(G=-1), av.EINVAL), (dict(G=65536), av.EUNSUPPORTED), (dict(mp=-1), av.EINVAL), (dict(T=-1), av.EINVAL),
    (dict(T=2 ** 29), av.EUNSUPPORTED), (dict(T=2 ** 24), av.EUNSUPPORTED),
    (dict(attn=_attn(num_q_heads=65536, num_kv_heads=65536)), av.EUNSUPPORTED), (dict(attn=_attn(max_blocks_per_seq=2 ** 27)), av.EUNSUPPORTED),
    (dict(q=None), av.EINVAL), (dict(gs=None), av.EINVAL), (dict(pl=None), av.EINVAL), (dict(out=None), av.EINVAL),
    (dict(kc=ctypes.c_void_p(0x1008)), av.EINVAL), (dict(vc=ctypes.c_void_p(0x1004)), av.EINVAL),
    (dict(ws=ctypes.c_void_p(0x1008)), av.EINVAL), (dict(ws=None), av.EWORKSPACE), (dict(size=100), av.EWORKSPACE),
    (dict(T=0, q=None), av.OK), (dict(attn=_attn(num_seqs=0), gs=None), av.OK),
])
def test_attention_shared(kw, want):
    assert _shared(**kw) == want


def _shared_size(params, T, mq, ms, G, mp):
    n = ctypes.c_size_t(0)
    assert av.library().verify_attention_shared_workspace_size(ctypes.byref(params), T, mq, ms, G, mp, ctypes.byref(n)) == av.OK
    return n.value


@pytest.mark.parametrize("dtype", [av.BF16, av.F32])
@pytest.mark.parametrize("heads", [(8, 8), (32, 8), (5, 1), (64, 1)])
@pytest.mark.parametrize("keys", [448, 1000, 3000, 6000])
def test_shared_workspace_covers_smaller_batches(keys, heads, dtype):
    sizes = {}
    for B in (1, 2, 7, 40, 300):
        for T in (1, 3, 4, 9, 10, 33, 40, 130, 300, 1000, 5000):
            for mq in (1, 9, 300):
                p = _attn(num_seqs=B, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=64, dtype=dtype,
                          max_blocks_per_seq=400)
                sizes[B, T, mq] = _shared_size(p, T, mq, keys, 2, 64)
    for (B, T, mq), size in sizes.items():
        assert all(other <= size for (b, t, m), other in sizes.items() if b <= B and t <= T and m == mq)


@pytest.mark.parametrize("dtype,d", [(av.BF16, 128), (av.F32, 128), (av.F32, 64)])
def test_shared_workspace_covers_smaller_batches_of_many_heads(dtype, d):
    """One row more may mean larger tiles, of every head."""
    for heads, mq in (((4096, 4096), 10 ** 6), ((4096, 4096), 20), ((8192, 4096), 33)):
        sizes = [_shared_size(_attn(num_seqs=2, num_q_heads=heads[0], num_kv_heads=heads[1], head_dim=d, dtype=dtype, max_blocks_per_seq=400),
                              T, mq, 5000, 1, 64) for T in range(1, 200)]
        assert sizes == sorted(sizes)


def test_short_requests_need_no_workspace():
    for keys, dtype, blocks, want in ((2048, av.BF16, 200, True), (2049, av.BF16, 200, False), (5000, av.BF16, 128, True),
                                      (448, av.F32, 200, True), (449, av.F32, 200, False), (5000, av.F32, 28, True)):
        size = lambda B, mq: _shared_size(_attn(num_seqs=B, max_blocks_per_seq=blocks, dtype=dtype), 300, mq, keys, 1, 64)
        assert (size(2, 3) == 0) == want
        assert size(1000, 3) > 0
    assert size(2, 3) == 0 and size(2, 10 ** 6) == 0 and size(70, 10 ** 6) > 0


def test_attention_shared_without_a_prefix_is_verify_attention():
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    p = _attn()
    av.library().verify_attention_workspace_size(ctypes.byref(p), 5, 3, 100, ctypes.byref(m))
    for groups, prefix in ((0, 64), (1, 15)):
        assert av.library().verify_attention_shared_workspace_size(ctypes.byref(p), 5, 3, 100, groups, prefix,
                                                                   ctypes.byref(n)) == av.OK
        assert n.value == m.value
        assert _shared(G=groups, mp=prefix, q=None) == av.EINVAL


def test_the_binding_refuses():
    i32 = torch.int32
    x, tok, qs = torch.zeros((5, 100)), torch.zeros(5, dtype=i32), torch.zeros(3, dtype=i32)
    counts, seen, one = torch.zeros((3, 100), dtype=i32), torch.zeros((3, 2, 4), dtype=i32), torch.ones(2)
    state = dict(counts=counts, seen=seen, repetition=one)
    bad = [
        dict(x=torch.zeros(5)), dict(x=torch.zeros((100, 5)).t()), dict(x=torch.zeros((1, 100)).expand(5, 100)),
        dict(qs=torch.zeros((3, 1), dtype=i32)), dict(tok=tok[:4], **state),
        dict(repetition=one), dict(**{**state, "seen": seen[:, :1]}), dict(**{**state, "counts": counts[:, :99]}),
        dict(**{**state, "repetition": torch.ones(3)}), dict(**state, slots=torch.zeros(3, dtype=i32)),
        dict(**{**state, "counts": counts[:1], "seen": seen[:1]}),  # two requests, one slot
        dict(bias_start=qs), dict(bias_tokens=tok, bias_values=one),
        dict(bias_start=qs, bias_tokens=tok, bias_values=torch.ones(4)),
        dict(mask=seen[:, 0]), dict(mask_rows=tok), dict(mask=seen[:, 0, :3].contiguous(), mask_rows=tok),
        dict(mask=seen[:, 0].contiguous(), mask_rows=tok[:3]), dict(out=torch.zeros((5, 99))),
        dict(x=torch.zeros((5, 100), dtype=torch.float16)),
    ]
    for kw in bad:
        kw = dict(kw)
        args = kw.pop("x", x), kw.pop("tok", tok), kw.pop("qs", qs)
        with pytest.raises((ValueError, TypeError)):
            av.verify_adjust_logits(*args, **kw)
    with pytest.raises(ValueError, match="device"):
        av.verify_adjust_logits(x, tok, qs)
    for args, kw in [((counts[0], seen, tok, qs), {}), ((counts, seen[0], tok, qs), {}), ((counts, seen, tok, qs[:0]), {}),
                     ((counts, seen, tok[None], qs), {}), ((counts, seen, tok, qs), dict(num_tokens=tok)),
                     ((counts[:1], seen[:1], tok, qs), {}), ((counts.long(), seen, tok, qs), {}),
                     ((counts, seen, tok, qs), {})]:
        with pytest.raises((ValueError, TypeError)):
            av.verify_count_tokens(*args, **kw)
    q, pos, freq = torch.zeros((5, 2, 64)), torch.zeros(5, dtype=i32), torch.zeros(32, dtype=torch.float64)
    for kw in (dict(q_weight=torch.ones(63)), dict(k_weight=torch.ones(64, dtype=torch.bfloat16)), {}):
        with pytest.raises((ValueError, TypeError)):
            av.verify_norm_rotary(q, None, pos, freq, **kw)


def test_the_binding_refuses_shared_attention():
    i32 = torch.int32
    kc, vc = torch.zeros((4, 2, 8, 16, 8), dtype=torch.bfloat16), torch.zeros((4, 2, 64, 16), dtype=torch.bfloat16)
    base = [torch.zeros((3, 4, 64), dtype=torch.bfloat16), kc, vc, torch.zeros((2, 2), dtype=i32), torch.zeros(2, dtype=i32),
            torch.zeros(3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32)]
    bounds = dict(max_q_len=2, max_seq_len=32, max_prefix_len=16)
    for at, t in [(0, base[0][0]), (1, kc[:, :1]), (2, vc.float()), (3, base[3][0]), (4, base[4][:1]), (5, base[5][:2]),
                  (6, base[6][:0]), (6, base[6].long()), (7, base[6]), (0, base[0])]:
        args = list(base)
        args[at] = t
        with pytest.raises((ValueError, TypeError)):
            av.verify_attention_shared(*args, **bounds)
    with pytest.raises(av.VerifyError):
        av.attention_shared_workspace_size(base[0], kc, base[3], num_groups=-1, **bounds)


def test_the_structs_agree_with_c():
    # 6 pointers, an int and its padding, 3 pointers, two ints, 2 pointers
    assert ctypes.sizeof(av.AdjustParams) == 6 * 8 + 8 + 3 * 8 + 8 + 2 * 8
    assert av.AdjustParams.num_masks.offset == 84 and av.AdjustParams.mask.offset == 88
