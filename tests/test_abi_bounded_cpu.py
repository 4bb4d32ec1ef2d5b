"""The rotary and bounded-cache calls on the host: every refusal comes before the GPU is
touched, from the library and from the binding."""
from __future__ import annotations

import ctypes
import os
import re

import pytest
import torch

import paper_2608_24004_amd as av

DUMMY = ctypes.c_void_p(0x1000)
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _attn(**kw):
    base = dict(num_seqs=2, num_q_heads=8, num_kv_heads=2, head_dim=128, block_size=16, max_blocks_per_seq=64,
                num_blocks=100, sliding_window=0, scale=0.0, dtype=av.BF16, kv_split_blocks=0)
    base.update(kw)
    return av.AttnParams(*[base[f] for f, _ in av.AttnParams._fields_])


def _rot(axes=(0,) * 64, **kw):
    p = av.RotaryParams(128, 128, 1, 0, 0.0, av.BF16)
    for f, a in enumerate(axes):
        p.axis[f] = a
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _rotary(p, T=3, hq=8, hkv=2, q=DUMMY, qs=1024, k=DUMMY, ks=256, pos=DUMMY, freq=DUMMY, qo=DUMMY, qos=1024, ko=DUMMY,
            kos=256):
    return av.library().verify_rotary(ctypes.byref(p) if p is not None else None, T, hq, hkv, q, qs, k, ks, pos, freq,
                                      qo, qos, ko, kos, None)


def test_the_header_and_the_binding_agree():
    src = open(os.path.join(ROOT, "include", "agentspec_verify.h")).read()
    assert int(re.search(r"#define VERIFY_ROTARY_MAX_AXES (\d+)", src)[1]) == av.ROTARY_MAX_AXES
    # the C struct: six 4-byte fields and 64 axis bytes
    assert ctypes.sizeof(av.RotaryParams) == 88 and av.RotaryParams.axis.offset == 24


@pytest.mark.parametrize("kw,want", [
    (dict(head_dim=96), av.EUNSUPPORTED),
    (dict(dtype=2), av.EUNSUPPORTED),
    (dict(rotary_dim=0), av.EINVAL),
    (dict(rotary_dim=7), av.EINVAL),
    (dict(rotary_dim=130), av.EINVAL),
    (dict(head_dim=64), av.EINVAL),          # rotary_dim 128 of 64
    (dict(num_axes=0), av.EINVAL),
    (dict(num_axes=5), av.EINVAL),
    (dict(interleaved=2), av.EINVAL),
    (dict(scale=-1.0), av.EINVAL),
    (dict(scale=float("inf")), av.EINVAL),
    (dict(scale=float("nan")), av.EINVAL),
    (dict(axes=[0] * 63 + [1]), av.EINVAL),  # an axis that is not there
])
def test_rotary_params(kw, want):
    assert _rotary(_rot(**kw)) == want
    args = (ctypes.byref(_attn()), ctypes.byref(_rot(**kw)), 3, DUMMY, 1024, DUMMY, 256, DUMMY, 256) + (DUMMY,) * 6
    assert av.library().verify_rotary_append(*args, 1024, DUMMY, DUMMY, None) == want


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), av.EINVAL), (dict(hq=0), av.EINVAL), (dict(hkv=-1), av.EINVAL),
    (dict(hq=40000, qs=1 << 40, qos=1 << 40), av.EUNSUPPORTED),
    (dict(q=None), av.EINVAL), (dict(pos=None), av.EINVAL), (dict(freq=None), av.EINVAL), (dict(qo=None), av.EINVAL),
    (dict(k=None), av.EINVAL), (dict(ko=None), av.EINVAL), (dict(hkv=0), av.EINVAL),
    (dict(qs=1023), av.EINVAL), (dict(qos=1000), av.EINVAL), (dict(ks=255), av.EINVAL), (dict(kos=-256), av.EINVAL),
    (dict(qs=2048), av.EINVAL),              # in place with two strides
    (dict(T=0, q=None, k=None, pos=None), av.OK),
])
def test_rotary_arguments(kw, want):
    assert _rotary(_rot(), **kw) == want
    assert _rotary(None) == av.EINVAL


@pytest.mark.parametrize("T", [(1 << 28) - 15, 1 << 28, 2 ** 31 - 15, 2 ** 31 - 1])
def test_rotary_of_more_rows_than_a_launch_holds(T):
    assert _rotary(_rot(), T=T) == av.EUNSUPPORTED
    for attn in (_attn(), _attn(num_seqs=0)):
        args = (ctypes.byref(attn), ctypes.byref(_rot()), T, DUMMY, 1024, DUMMY, 256, DUMMY, 256) + (DUMMY,) * 6
        assert av.library().verify_rotary_append(*args, 1024, DUMMY, DUMMY, None) == av.EUNSUPPORTED


def test_rotary_append_arguments():
    lib = av.library()

    def call(attn=None, rot=None, T=3, strides=(1024, 256, 256, 1024), ptrs=None, kc=DUMMY, vc=DUMMY):
        p = [DUMMY] * 9
        for k, v in (ptrs or {}).items():
            p[k] = v
        q, k, v, pos, freq, bt, sl, qs, qo = p
        return lib.verify_rotary_append(ctypes.byref(attn or _attn()), ctypes.byref(rot or _rot()), T, q, strides[0], k,
                                        strides[1], v, strides[2], pos, freq, bt, sl, qs, qo, strides[3], kc, vc, None)
    for x in range(9):
        assert call(ptrs={x: None}) == av.EINVAL
    assert call(kc=None) == call(vc=None) == av.EINVAL
    assert call(kc=ctypes.c_void_p(0x1008)) == av.EINVAL      # not 16-byte aligned
    assert call(rot=_rot(dtype=av.F32)) == av.EINVAL          # another type than the cache's
    assert call(attn=_attn(head_dim=64)) == av.EINVAL
    assert call(attn=_attn(block_size=32)) == av.EUNSUPPORTED
    assert call(strides=(1024, 256, 255, 1024)) == av.EINVAL
    assert call(T=0, ptrs={0: None}) == av.OK


def _weights(attn, T=18, mq=9, ms=1000, ptrs=None, decay=1.0, ws=DUMMY, have=1 << 30):
    p = [DUMMY] * 10  # q, kc, bt, sl, qs, rows, tokens, sinks, weights, order
    for k, v in (ptrs or {}).items():
        p[k] = v
    return av.library().verify_key_weights(ctypes.byref(attn) if attn is not None else None, T, mq, ms, *p[:8], decay,
                                           *p[8:], ws, have, None)


def test_key_weights_arguments():
    size = ctypes.c_size_t(0)
    query = av.library().verify_key_weights_workspace_size
    assert query(ctypes.byref(_attn()), 18, 9, 1000, ctypes.byref(size)) == av.OK and size.value > 0
    assert query(ctypes.byref(_attn()), 18, 9, 1000, None) == av.EINVAL
    for kw, want in ((dict(sliding_window=128), av.EUNSUPPORTED), (dict(head_dim=80), av.EUNSUPPORTED),
                     (dict(num_q_heads=7), av.EINVAL), (dict(num_seqs=-1), av.EINVAL), (dict(scale=-1.0), av.EINVAL)):
        assert query(ctypes.byref(_attn(**kw)), 18, 9, 1000, ctypes.byref(size)) == want
        assert _weights(_attn(**kw)) == want
    assert _weights(None) == av.EINVAL
    for x in (0, 1, 2, 3, 4, 8, 9):
        assert _weights(_attn(), ptrs={x: None}) == av.EINVAL
    assert _weights(_attn(), ptrs={1: ctypes.c_void_p(0x1004)}) == av.EINVAL
    for decay in (-0.5, float("nan"), float("inf")):
        assert _weights(_attn(), decay=decay) == av.EINVAL
    for kw in (dict(T=-1), dict(mq=-1), dict(ms=-1)):
        assert _weights(_attn(), **kw) == av.EINVAL
    assert _weights(_attn(), have=0) == _weights(_attn(), ws=None) == av.EWORKSPACE
    # a grid that no launch holds
    assert _weights(_attn(num_q_heads=4096, num_kv_heads=4096, max_blocks_per_seq=1 << 26), ms=(1 << 30)) == av.EUNSUPPORTED
    # a group that the row arithmetic does not hold
    assert _weights(_attn(num_q_heads=8192, num_kv_heads=1), T=64) == av.EUNSUPPORTED
    for T in (1 << 30, 2 ** 31 - 1):
        assert _weights(_attn(num_q_heads=2, num_kv_heads=2), T=T) == av.EUNSUPPORTED
        assert _weights(_attn(num_q_heads=4, num_kv_heads=2), T=T // 2 + 1) == av.EUNSUPPORTED
    assert _weights(_attn(), ws=ctypes.c_void_p(0x1008)) == av.EINVAL
    assert _weights(_attn(num_seqs=0), T=0, have=0, ws=None) == av.OK


@pytest.mark.parametrize("dtype", [av.BF16, av.F32])
@pytest.mark.parametrize("hq,hkv,d,mq,ms", [(32, 8, 128, 9, 16384), (8, 8, 128, 1, 5000), (64, 1, 64, 1, 4000),
                                            (32, 2, 128, 200, 4000), (8, 1, 128, 9, 131072), (32, 8, 64, 600, 900)])
def test_key_weights_workspace_covers_fewer_requests_with_as_many_rows(dtype, hq, hkv, d, mq, ms):
    """The size asked for a batch serves every batch of fewer requests and rows, also
    one with more rows than its requests announce (max_q_len only sizes the launch).  A
    cache of no blocks: the call ends after its checks."""
    size = ctypes.c_size_t(0)
    attn = lambda B: _attn(num_seqs=B, num_q_heads=hq, num_kv_heads=hkv, head_dim=d, dtype=dtype, num_blocks=0,
                           max_blocks_per_seq=-(-ms // 16))
    for B, T in ((32, 32 * mq), (32, 7), (5, 500), (1, 1)):
        assert av.library().verify_key_weights_workspace_size(ctypes.byref(attn(B)), T, mq, ms,
                                                              ctypes.byref(size)) == av.OK
        for b in sorted({1, 2, 3, (B + 1) // 2, B}):
            for t in sorted({1, T // 3, T - 1, T}):
                if b <= B:
                    assert _weights(attn(b), T=t, mq=mq, ms=ms, have=size.value) == av.OK, (B, T, b, t)


def _plan(attn, ms=1000, keys=100, first=4, recent=10, ptrs=None, ws=DUMMY, have=1 << 30):
    p = [DUMMY] * 7  # weights, order, bt, sl, tokens, source, lens
    for k, v in (ptrs or {}).items():
        p[k] = v
    return av.library().verify_evict_plan(ctypes.byref(attn) if attn is not None else None, ms, keys, first, recent, *p,
                                          ws, have, None)


def test_evict_plan_arguments():
    query = av.library().verify_evict_plan_workspace_size
    size = ctypes.c_size_t(0)
    assert query(ctypes.byref(_attn()), 1000, 100, ctypes.byref(size)) == av.OK
    assert size.value == 0                                    # a workgroup's own memory holds it
    long = _attn(max_blocks_per_seq=4096)
    assert query(ctypes.byref(long), 40000, 100, ctypes.byref(size)) == av.OK and size.value > 0
    need = size.value
    assert query(ctypes.byref(long), 40000, 40000, ctypes.byref(size)) == av.OK and size.value == 0  # nobody exceeds it
    far = _attn(max_blocks_per_seq=1 << 25)
    assert query(ctypes.byref(far), (1 << 24) + 1, 100, ctypes.byref(size)) == av.EUNSUPPORTED
    assert _plan(far, ms=(1 << 24) + 1) == av.EUNSUPPORTED
    assert query(ctypes.byref(_attn()), 1000, 100, None) == av.EINVAL
    assert query(None, 1000, 100, ctypes.byref(size)) == av.EINVAL
    assert _plan(None) == av.EINVAL
    for kw in (dict(keys=0), dict(keys=-5), dict(first=-1), dict(recent=-1), dict(first=60, recent=41), dict(ms=-1),
               dict(first=2 ** 31 - 1, recent=2 ** 31 - 1)):
        assert _plan(_attn(), **kw) == av.EINVAL
    for x in (0, 2, 3, 5, 6):
        assert _plan(_attn(), ptrs={x: None}) == av.EINVAL
    assert _plan(_attn(sliding_window=64)) == av.EUNSUPPORTED
    for x in (0, 1):
        assert _plan(_attn(), ptrs={x: ctypes.c_void_p(0x1004)}) == av.EINVAL
    for heads in (1 << 16, 1 << 17):
        many = _attn(num_q_heads=heads, num_kv_heads=heads, max_blocks_per_seq=4096)
        for ms in (1000, 40000):
            assert query(ctypes.byref(many), ms, 100, ctypes.byref(size)) == _plan(many, ms=ms) == av.EUNSUPPORTED
    assert _plan(long, ms=40000, ws=ctypes.c_void_p(0x1008)) == av.EINVAL
    assert _plan(long, ms=40000, have=need - 1) == _plan(long, ms=40000, ws=None) == av.EWORKSPACE
    assert _plan(_attn(num_seqs=0), have=0, ws=None) == av.OK


def test_kv_compact_arguments():
    def call(attn, keys=100, ptrs=None):
        p = [DUMMY] * 7  # bt, source, lens, kc, vc, weights, order
        for k, v in (ptrs or {}).items():
            p[k] = v
        return av.library().verify_kv_compact(ctypes.byref(attn) if attn is not None else None, keys, *p, None)
    assert call(None) == av.EINVAL
    for x in range(5):
        assert call(_attn(), ptrs={x: None}) == av.EINVAL
    for x in (3, 4):
        assert call(_attn(), ptrs={x: ctypes.c_void_p(0x1002)}) == av.EINVAL
    assert call(_attn(), keys=0) == av.EINVAL
    assert call(_attn(sliding_window=1)) == av.EUNSUPPORTED
    assert call(_attn(num_seqs=0)) == av.OK


def _t(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype)


def test_the_binding_refuses():
    """Shapes, types and places of tensors, before any call."""
    i32, f64 = torch.int32, torch.float64
    q, k, pos, freq = _t(3, 4, 64), _t(3, 2, 64), _t(2, 3, dtype=i32), _t(32, dtype=f64)
    axes = [0, 1] * 16
    rot = lambda *a, **kw: av.verify_rotary(*a, **dict(dict(axes=axes), **kw))
    with pytest.raises(ValueError, match="device tensor"):
        rot(q, k, pos, freq)
    with pytest.raises(ValueError, match="axes"):
        rot(q, k, pos, freq, axes=None)
    with pytest.raises(ValueError, match="axes"):
        rot(q, k, pos, freq, axes=[0, 1])
    with pytest.raises(ValueError, match="axes"):
        rot(q, k, pos, freq, axes=[2] * 32)
    with pytest.raises(ValueError, match="axes"):
        rot(q, k, pos, freq, axes=[-1] * 32)
    with pytest.raises(ValueError, match="positions"):
        rot(q, k, _t(2, 4, dtype=i32), freq)
    with pytest.raises(TypeError, match="positions"):
        rot(q, k, _t(2, 3, dtype=torch.int64), freq)
    with pytest.raises(TypeError, match="inv_freq"):
        rot(q, k, pos, freq.float())
    with pytest.raises(ValueError, match="rotary_dim"):
        rot(q, k, pos, _t(33, dtype=f64), axes=[0] * 33)
    with pytest.raises(TypeError, match="k must be"):
        rot(q, k.float(), pos, freq)
    with pytest.raises(ValueError, match="k must have shape"):
        rot(q, _t(2, 2, 64), pos, freq)
    with pytest.raises(ValueError, match="adjacent"):
        rot(_t(3, 64, 4).transpose(1, 2), k, pos, freq)
    with pytest.raises(ValueError, match="adjacent"):
        rot(q, _t(3, 4, 64)[:, ::2], pos, freq)
    with pytest.raises(TypeError, match="storage dtype"):
        rot(q.half(), k.half(), pos, freq)
    kc, vc = _t(5, 2, 8, 16, 8), _t(5, 2, 64, 16)
    bt, sl, qs = _t(1, 3, dtype=i32), _t(1, dtype=i32), _t(2, dtype=i32)
    app = lambda *a: av.verify_rotary_append(*a, axes=axes)
    with pytest.raises(ValueError, match="device tensor"):
        app(q, k, k, pos, freq, kc, vc, bt, sl, qs)
    with pytest.raises(ValueError, match="v_new"):
        app(q, k, _t(3, 3, 64), pos, freq, kc, vc, bt, sl, qs)
    with pytest.raises(ValueError, match="q_start"):
        app(q, k, k, pos, freq, kc, vc, bt, sl, _t(3, dtype=i32))
    w, o = _t(5, 2, 16, dtype=torch.float32), _t(5, 2, 16, dtype=i32)
    bounds = dict(max_q_len=3, max_seq_len=40)
    wgt = lambda *a, **kw: av.verify_key_weights(*a, **dict(bounds, **kw))
    with pytest.raises(ValueError, match="device tensor"):
        wgt(q, kc, w, o, bt, sl, qs)
    with pytest.raises(ValueError, match="key_weights"):
        wgt(q, kc, w[:4], o, bt, sl, qs)
    with pytest.raises(TypeError, match="key_order"):
        wgt(q, kc, w, o.long(), bt, sl, qs)
    with pytest.raises(ValueError, match="num_rows"):
        wgt(q, kc, w, o, bt, sl, qs, num_rows=_t(2, dtype=i32))
    with pytest.raises(TypeError, match="k_cache"):
        wgt(q, kc.float(), w, o, bt, sl, qs)
    with pytest.raises(TypeError, match="sinks"):
        wgt(q, kc, w, o, bt, sl, qs, sinks=_t(4))
    with pytest.raises(ValueError, match="is required"):
        wgt(q, kc, w, o, bt, None, qs)
    plan = lambda *a, **kw: av.verify_evict_plan(*a, **dict(dict(max_keys=8, max_seq_len=40), **kw))
    with pytest.raises(ValueError, match="device tensor"):
        plan(w, o, bt, sl)
    with pytest.raises(ValueError, match="source"):
        plan(w, o, bt, sl, source=_t(1, 2, 7, dtype=i32))
    with pytest.raises(ValueError, match="key_weights"):
        plan(_t(5, 2, 8, dtype=torch.float32), o, bt, sl)
    with pytest.raises(av.VerifyError, match="invalid argument"):
        plan(w, o, bt, sl, max_keys=0)
    src = _t(1, 2, 8, dtype=i32)
    with pytest.raises(ValueError, match="device tensor"):
        av.verify_kv_compact(kc, vc, bt, src, sl)
    with pytest.raises(ValueError, match="v_cache"):
        av.verify_kv_compact(kc, _t(5, 2, 32, 16), bt, src, sl)
    with pytest.raises(ValueError, match="source"):
        av.verify_kv_compact(kc, vc, bt, _t(2, 2, 8, dtype=i32), sl)
    with pytest.raises(ValueError, match="new_lens"):
        av.verify_kv_compact(kc, vc, bt, src, _t(2, dtype=i32))
