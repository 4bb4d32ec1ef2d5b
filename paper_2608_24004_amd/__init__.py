"""MI355X-native batched speculative-verification step (AgentSpec hot path).

Thin ctypes binding over the C ABI in ``include/agentspec_verify.h``: argument
marshalling only.  Every step of the verify pass runs in the HIP kernels of
``libagentspec_verify.so``; PyTorch supplies device memory and the stream.
If the library is missing, every entry point raises -- there is no fallback.

    verify_attention(...)      paged multi-query GQA attention of all scored rows
    verify_accept(...)         vocabulary argmax + greedy acceptance of the drafts
    verify_lmhead_accept(...)  the same acceptance fed by the LM head, logits
                               never stored
    verify_accept_sampled(...), verify_budget(...), verify_kv_append(...)
    verify_attention_append(...) the append and the attention in one launch
    check_batch(...)           the batch descriptor's preconditions, checked on
                               the device (the calls above take ``check=True``,
                               or every call does with AGENTSPEC_VERIFY_CHECK=1)
    check_groups(...)          those of groups of requests, which
                               verify_attention_shared checks beside them
    verify_rotary(...), verify_rotary_append(...)
                               queries and keys rotated to positions on one or
                               several axes, alone or with the append
    verify_norm_rotary(...), verify_norm_rotary_append(...)
                               the same behind a norm of each head's query and key
    verify_attention_shared(...)
                               verify_attention where groups of requests begin with the
                               same cached tokens, whose keys are read once
    verify_adjust_logits(...), verify_count_tokens(...)
                               penalties, biases and grammar masks on the logits, and
                               the token counts that the penalties read
    verify_key_weights(...), verify_evict_plan(...), verify_kv_compact(...)
                               a bound on a request's cached keys: the attention
                               weight each has gathered, the keys to keep, their
                               moves
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

from .build import LIB_PATH

__all__ = ["verify_attention", "verify_accept", "verify_accept_noalloc", "verify_accept_sampled",
           "verify_lmhead_accept",
           "verify_budget", "verify_kv_append", "verify_attention_append",
           "attention_workspace_size", "attention_plan",
           "accept_workspace_size",
           "lmhead_accept_workspace_size", "verify_rotary", "verify_rotary_append",
           "verify_norm_rotary", "verify_norm_rotary_append", "verify_adjust_logits", "verify_count_tokens",
           "verify_attention_shared", "attention_shared_workspace_size",
           "verify_key_weights", "verify_evict_plan", "verify_kv_compact",
           "key_weights_workspace_size", "evict_plan_workspace_size", "check_batch", "check_groups", "BatchError", "VerifyError", "library",
           "abi_version", "F32", "BF16"]

OK, EINVAL, EUNSUPPORTED, EWORKSPACE, EHIP = 0, -1, -2, -3, -4
NOALLOC_SCRATCH_BYTES = 4 << 20  # VERIFY_NOALLOC_SCRATCH_BYTES of the C header
F32, BF16 = 0, 1
# verify_check_batch's counts, in the order of VERIFY_CHECK_ROWS .. _BLOCK_ID,
# then the first offending request (VERIFY_CHECK_FIRST)
CHECK_KINDS = ("rows", "q_len", "short_seq", "long_seq", "block_id")
CHECK_COUNTS = 6
# verify_check_groups' counts, likewise, then the first offending group
CHECK_GROUPS_KINDS = ("bounds", "table")
ROTARY_MAX_AXES = 4  # VERIFY_ROTARY_MAX_AXES
CHECK_BY_DEFAULT = os.environ.get("AGENTSPEC_VERIFY_CHECK", "0") == "1"


class VerifyError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, _status_string(status), status))


class BatchError(ValueError):
    """A batch descriptor that fails verify_check_batch: ``counts`` maps each
    kind in CHECK_KINDS to its number of offending requests, ``first`` is the
    lowest offending request.  Or one whose groups fail verify_check_groups: then the
    kinds are CHECK_GROUPS_KINDS and ``first`` is the lowest offending group."""

    def __init__(self, where: str, counts: dict, first: int, of: str = "request"):
        self.counts, self.first = counts, first
        bad = ", ".join("%s %d" % (k, v) for k, v in counts.items() if v)
        super().__init__("%s: bad batch descriptor (%s; first %s %d)" % (where, bad, of, first))


class AttnParams(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block_size", ctypes.c_int32),
        ("max_blocks_per_seq", ctypes.c_int32),
        ("num_blocks", ctypes.c_int32),
        ("sliding_window", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("dtype", ctypes.c_int32),
        ("kv_split_blocks", ctypes.c_int32),
    ]


class RotaryParams(ctypes.Structure):
    _fields_ = [
        ("head_dim", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32),
        ("num_axes", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("dtype", ctypes.c_int32),
        ("axis", ctypes.c_uint8 * 64),
    ]


class AdjustParams(ctypes.Structure):
    _fields_ = [
        ("repetition", ctypes.c_void_p),
        ("frequency", ctypes.c_void_p),
        ("presence", ctypes.c_void_p),
        ("counts", ctypes.c_void_p),
        ("seen", ctypes.c_void_p),
        ("slots", ctypes.c_void_p),
        ("num_slots", ctypes.c_int32),
        ("bias_start", ctypes.c_void_p),
        ("bias_tokens", ctypes.c_void_p),
        ("bias_values", ctypes.c_void_p),
        ("num_biases", ctypes.c_int32),
        ("num_masks", ctypes.c_int32),
        ("mask", ctypes.c_void_p),
        ("mask_rows", ctypes.c_void_p),
    ]


_lib = None


def library(path: Optional[str] = None):
    """Load (once) and return the ctypes handle of the HIP library."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    path = path or os.environ.get("AGENTSPEC_VERIFY_LIB", LIB_PATH)
    if not os.path.exists(path):
        raise RuntimeError("verify library not built: %s is missing "
                           "(run `python -m paper_2608_24004_amd.build`)" % path)
    lib = ctypes.CDLL(path)
    i32, i64, vp, sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t
    P = ctypes.POINTER(AttnParams)
    lib.verify_attention_workspace_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(sz)]
    lib.verify_attention_workspace_size.restype = ctypes.c_int
    lib.verify_attention.argtypes = [P, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.verify_attention.restype = ctypes.c_int
    lib.verify_attention_plan.argtypes = [P, i32, i32, i32, ctypes.POINTER(i32)]
    lib.verify_attention_plan.restype = ctypes.c_int
    lib.verify_kv_append.argtypes = [P, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.verify_attention_append.argtypes = [P, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                            vp, sz, vp]
    lib.verify_attention_append.restype = ctypes.c_int
    lib.verify_kv_append.restype = ctypes.c_int
    lib.verify_accept_workspace_size.argtypes = [i32, i32, i64, i32, ctypes.POINTER(sz)]
    lib.verify_accept_workspace_size.restype = ctypes.c_int
    lib.verify_accept.argtypes = [i32, i32, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.verify_accept.restype = ctypes.c_int
    lib.verify_accept_noalloc.argtypes = [i32, i32, i64, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.verify_accept_noalloc.restype = ctypes.c_int
    lib.verify_accept_sampled.argtypes = [i32, i32, i64, i64, i32, vp, vp, vp, ctypes.c_float,
                                          ctypes.c_uint64, ctypes.c_uint32, vp, vp, vp, vp, vp, sz, vp]
    lib.verify_accept_sampled.restype = ctypes.c_int
    f64 = ctypes.c_double
    lib.verify_lmhead_accept_workspace_size.argtypes = [i32, i32, i32, i64, i32, ctypes.POINTER(sz)]
    lib.verify_lmhead_accept_workspace_size.restype = ctypes.c_int
    lib.verify_lmhead_accept.argtypes = [i32, i32, i32, i64, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp,
                                         sz, vp]
    lib.verify_lmhead_accept.restype = ctypes.c_int
    lib.verify_budget.argtypes = [i32, i32, i32, vp, vp, vp, vp, vp, f64, f64, vp, vp, vp, vp, vp, vp,
                                  vp, i64, vp, vp]
    lib.verify_budget.restype = ctypes.c_int
    lib.verify_check_batch.argtypes = [i32, i32, i32, vp, P, i32, vp, vp, vp, vp]
    lib.verify_check_batch.restype = ctypes.c_int
    lib.verify_check_groups.argtypes = [P, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.verify_check_groups.restype = ctypes.c_int
    RP, f32 = ctypes.POINTER(RotaryParams), ctypes.c_float
    lib.verify_rotary.argtypes = [RP, i32, i32, i32, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, vp]
    lib.verify_rotary.restype = ctypes.c_int
    lib.verify_rotary_append.argtypes = [P, RP, i32, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp,
                                         vp, vp]
    lib.verify_rotary_append.restype = ctypes.c_int
    lib.verify_norm_rotary.argtypes = [RP, i32, i32, i32, vp, i64, vp, i64, vp, vp, f32, vp, vp, vp, i64, vp, i64, vp]
    lib.verify_norm_rotary.restype = ctypes.c_int
    lib.verify_norm_rotary_append.argtypes = [P, RP, i32, vp, i64, vp, i64, vp, i64, vp, vp, f32, vp, vp, vp, vp, vp,
                                              vp, i64, vp, vp, vp]
    lib.verify_norm_rotary_append.restype = ctypes.c_int
    lib.verify_attention_shared_workspace_size.argtypes = [P, i32, i32, i32, i32, i32, ctypes.POINTER(sz)]
    lib.verify_attention_shared_workspace_size.restype = ctypes.c_int
    lib.verify_attention_shared.argtypes = [P, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz,
                                            vp]
    lib.verify_attention_shared.restype = ctypes.c_int
    lib.verify_adjust_logits.argtypes = [i32, i32, i64, i64, i32, vp, vp, vp, ctypes.POINTER(AdjustParams), vp, i64, vp]
    lib.verify_adjust_logits.restype = ctypes.c_int
    lib.verify_count_tokens.argtypes = [i32, i32, i64, i32, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.verify_count_tokens.restype = ctypes.c_int
    lib.verify_key_weights_workspace_size.argtypes = [P, i32, i32, i32, ctypes.POINTER(sz)]
    lib.verify_key_weights_workspace_size.restype = ctypes.c_int
    lib.verify_key_weights.argtypes = [P, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, f32, vp, vp, vp, sz, vp]
    lib.verify_key_weights.restype = ctypes.c_int
    lib.verify_evict_plan_workspace_size.argtypes = [P, i32, i32, ctypes.POINTER(sz)]
    lib.verify_evict_plan_workspace_size.restype = ctypes.c_int
    lib.verify_evict_plan.argtypes = [P, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.verify_evict_plan.restype = ctypes.c_int
    lib.verify_kv_compact.argtypes = [P, i32, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.verify_kv_compact.restype = ctypes.c_int
    lib.verify_status_string.argtypes = [ctypes.c_int]
    lib.verify_status_string.restype = ctypes.c_char_p
    lib.verify_abi_version.argtypes = []
    lib.verify_abi_version.restype = ctypes.c_int
    if path == LIB_PATH or _lib is None:
        _lib = lib
    return lib


def _status_string(status: int) -> str:
    try:
        return library().verify_status_string(status).decode()
    except Exception:
        return "status %d" % status


def abi_version() -> int:
    return int(library().verify_abi_version())


def _check(status: int, where: str):
    if status != OK:
        raise VerifyError(status, where)


_dtype_codes = {}


def _dtype_code(t) -> int:
    code = _dtype_codes.get(t.dtype)
    if code is not None:
        return code
    import torch
    _dtype_codes.update({torch.bfloat16: BF16, torch.float32: F32})
    if t.dtype not in _dtype_codes:
        raise TypeError("unsupported storage dtype %s (bf16 or fp32)" % t.dtype)
    return _dtype_codes[t.dtype]


def _dev_ptr(t, name, dtype=None):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


def _expect(t, name, shape=None, dtype=None, device=None):
    """Check a caller tensor before its pointer crosses the ABI.

    The kernels index device memory by the sizes passed beside the pointers,
    so a tensor smaller than those sizes would be read or written out of
    bounds, and one on another device would be read through the wrong
    address space."""
    if t is None:
        raise ValueError("%s is required" % name)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if device is not None and t.device != device:
        raise ValueError("%s is on %s, the call runs on %s" % (name, t.device, device))


def _arg(t, name, shape, dtype, idx, device):
    """Device address of a required caller tensor, checked by _expect and
    _dev_ptr.  The tests that a good tensor passes are made here first, in one
    go: with some ten tensors per call the full checks took as long as the
    kernels of a small call (one request's attention: 21 us on the host, 14 us
    on the GPU)."""
    if (t is not None and t.dtype is dtype and t.get_device() == idx >= 0 and t.is_contiguous()
            and (shape is None or t.shape == shape)):
        return t.data_ptr()
    _expect(t, name, shape, dtype, device)
    # a call on tensors in host memory is refused by its first tensor, once
    # all are checked
    return _dev_ptr(t, name, dtype) if idx >= 0 else None


def _workspace_arg(workspace, idx, device):
    """Address and bytes of a caller's workspace."""
    if workspace is None:
        return None, 0
    return (_arg(workspace, "workspace", None, workspace.dtype, idx, device),
            workspace.numel() * workspace.element_size())


_attn_kept = {}


def _layer_args(Hq, D, dtype, esize, idx, dev, k_cache, v_cache, block_tables, seq_lens, q_start, own=True):
    """Addresses of a layer's cache and batch descriptor, and its AttnParams
    (sliding_window, scale and kv_split_blocks 0): the caller's own, or one kept for
    every call of the same sizes, which nobody may change.  A batch of no requests may
    come without seq_lens and q_start; the call refuses their absence otherwise."""
    import torch
    i32 = torch.int32
    if k_cache.dim() != 5:
        raise ValueError("k_cache must be [num_blocks, Hkv, D/x, 16, x], got %s" % (tuple(k_cache.shape),))
    nb, hkv = k_cache.shape[0], k_cache.shape[1]
    x = 16 // esize
    ptrs = [_arg(k_cache, "k_cache", (nb, hkv, D // x, 16, x), dtype, idx, dev),
            _arg(v_cache, "v_cache", (nb, hkv, D, 16), dtype, idx, dev)]
    if block_tables.dim() != 2:
        raise ValueError("block_tables must be [B, max_blocks], got %s" % (tuple(block_tables.shape),))
    B, max_blocks = block_tables.shape
    ptrs += [_arg(block_tables, "block_tables", None, i32, idx, dev),
             None if seq_lens is None else _arg(seq_lens, "seq_lens", (B,), i32, idx, dev),
             None if q_start is None else _arg(q_start, "q_start", (B + 1,), i32, idx, dev)]
    key = (B, Hq, hkv, D, 16, max_blocks, nb, 0, 0.0, _dtype_code(k_cache), 0)
    if own:
        return ptrs, AttnParams(*key)
    params = _attn_kept.get(key)
    if params is None:
        if len(_attn_kept) > 64:
            _attn_kept.clear()
        params = _attn_kept[key] = AttnParams(*key)
    return ptrs, params


# torch.cuda.current_stream builds a Stream object per call (2 us)
_raw_stream = None


def _stream_ptr(stream, device):
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda idx: torch.cuda.current_stream(idx).cuda_stream)
    return _raw_stream(device.index)


def _attn_params(q, k_cache, block_tables, sliding_window, scale, kv_split_blocks):
    T, Hq, D = q.shape
    params = AttnParams()
    params.num_seqs = block_tables.shape[0]
    params.num_q_heads = Hq
    params.num_kv_heads = k_cache.shape[1]
    params.head_dim = D
    params.block_size = k_cache.shape[3]
    params.max_blocks_per_seq = block_tables.shape[1]
    params.num_blocks = k_cache.shape[0]
    params.sliding_window = int(sliding_window)
    params.scale = float(scale)
    params.dtype = _dtype_code(q)
    params.kv_split_blocks = int(kv_split_blocks)
    return params


def check_batch(q_start, total_q: int, *, max_q_len: int = 0, seq_lens=None, block_tables=None,
                num_blocks: int = 0, max_seq_len: int = 0, sliding_window: int = 0, stream=None):
    """The batch descriptor's preconditions, checked on the device by
    verify_check_batch.  Waits for the call's stream and returns (counts,
    first): offending requests per kind of CHECK_KINDS, and the lowest
    offending request (-1 if none).

    Only q_start (and n_i <= max_q_len when max_q_len > 0) is checked unless
    seq_lens is given; then also n_i <= S_i <= max_seq_len, and with
    block_tables and num_blocks the ids of every block the rows can read
    (keys from the first row's window start, sliding_window > 0, or 0)."""
    import torch
    i32 = torch.int32
    if q_start.dim() != 1 or q_start.shape[0] < 1:
        raise ValueError("q_start must be [B + 1], got %s" % (tuple(q_start.shape),))
    B = q_start.shape[0] - 1
    dev = q_start.device
    params = None
    if seq_lens is not None:
        _expect(seq_lens, "seq_lens", (B,), i32, dev)
        params = AttnParams(num_seqs=B, block_size=16, num_blocks=int(num_blocks),
                            sliding_window=int(sliding_window),
                            max_blocks_per_seq=(1 << 31) // 16 - 1)
        if block_tables is not None:
            if block_tables.dim() != 2 or block_tables.shape[0] != B or block_tables.shape[1] < 1:
                raise ValueError("block_tables must be [B, max_blocks], got %s"
                                 % (tuple(block_tables.shape),))
            _expect(block_tables, "block_tables", None, i32, dev)
            params.max_blocks_per_seq = block_tables.shape[1]
    elif block_tables is not None:
        raise ValueError("block_tables are checked against seq_lens, which is missing")
    counts = torch.empty(CHECK_COUNTS, dtype=i32, device=dev)
    rc = library().verify_check_batch(
        B, int(total_q), int(max_q_len), _dev_ptr(q_start, "q_start", i32),
        ctypes.byref(params) if params is not None else None, int(max_seq_len),
        _dev_ptr(seq_lens, "seq_lens", i32), _dev_ptr(block_tables, "block_tables", i32),
        _dev_ptr(counts, "counts", i32), _stream_ptr(stream, dev))
    _check(rc, "verify_check_batch")
    (stream if stream is not None else torch.cuda.current_stream(dev)).synchronize()
    c = counts.cpu().tolist()
    return dict(zip(CHECK_KINDS, c[:len(CHECK_KINDS)])), (c[-1] if c[-1] != 2 ** 31 - 1 else -1)


def check_groups(group_start, prefix_lens, seq_lens, block_tables, *, max_prefix_len: int, max_seq_len: int, stream=None):
    """The preconditions of groups of requests (see verify_attention_shared), checked on
    the device by verify_check_groups: that group_start ascends within the batch, and that
    the requests of a group name the same blocks for their common prefix.  Waits for the
    call's stream and returns (counts, first): offenders per kind of CHECK_GROUPS_KINDS,
    groups and requests, and the lowest group with one (-1 if none)."""
    import torch
    i32, dev = torch.int32, group_start.device
    if group_start.dim() != 1 or group_start.shape[0] < 1:
        raise ValueError("group_start must be [G + 1], got %s" % (tuple(group_start.shape),))
    if block_tables.dim() != 2 or block_tables.shape[1] < 1:
        raise ValueError("block_tables must be [B, max_blocks], got %s" % (tuple(block_tables.shape),))
    B, G = block_tables.shape[0], group_start.shape[0] - 1
    _expect(group_start, "group_start", None, i32, dev)
    _expect(prefix_lens, "prefix_lens", (G,), i32, dev)
    _expect(seq_lens, "seq_lens", (B,), i32, dev)
    _expect(block_tables, "block_tables", None, i32, dev)
    params = AttnParams(num_seqs=B, block_size=16, max_blocks_per_seq=block_tables.shape[1])
    arrays = [_dev_ptr(group_start, "group_start"), _dev_ptr(prefix_lens, "prefix_lens"), _dev_ptr(seq_lens, "seq_lens"),
              _dev_ptr(block_tables, "block_tables")]
    counts = torch.empty(len(CHECK_GROUPS_KINDS) + 1, dtype=i32, device=dev)
    _launch("verify_check_groups", dev.index, ctypes.byref(params), int(max_seq_len), G, int(max_prefix_len), *arrays,
            counts.data_ptr(), _stream_ptr(stream, dev))
    (stream if stream is not None else torch.cuda.current_stream(dev)).synchronize()
    c = counts.cpu().tolist()
    return dict(zip(CHECK_GROUPS_KINDS, c)), (c[-1] if c[-1] != 2 ** 31 - 1 else -1)


def _checked(check, where, **kw):
    """Raise BatchError before `where` launches anything if the descriptor
    fails verify_check_batch (with check=True, or by default when
    AGENTSPEC_VERIFY_CHECK=1)."""
    if not (CHECK_BY_DEFAULT if check is None else check):
        return
    counts, first = check_batch(**kw)
    if any(counts.values()):
        raise BatchError(where, counts, first)


def attention_workspace_size(q, k_cache, block_tables, *, max_q_len: int, max_seq_len: int,
                             sliding_window: int = 0, scale: float = 0.0,
                             kv_split_blocks: int = 0) -> int:
    params = _attn_params(q, k_cache, block_tables, sliding_window, scale, kv_split_blocks)
    n = ctypes.c_size_t(0)
    _check(library().verify_attention_workspace_size(ctypes.byref(params), q.shape[0], int(max_q_len),
                                                     int(max_seq_len), ctypes.byref(n)),
           "verify_attention_workspace_size")
    return int(n.value)


PLAN_INFO = 11  # entries of verify_attention_plan's info array


def attention_plan(q, k_cache, block_tables, *, max_q_len: int, max_seq_len: int,
                   sliding_window: int = 0, scale: float = 0.0, kv_split_blocks: int = 0) -> dict:
    """The work decomposition verify_attention would use (nothing is launched)."""
    p = _attn_params(q, k_cache, block_tables, sliding_window, scale, kv_split_blocks)
    info = (ctypes.c_int32 * PLAN_INFO)()
    _check(library().verify_attention_plan(ctypes.byref(p), int(q.shape[0]), int(max_q_len),
                                           int(max_seq_len), info), "verify_attention_plan")
    v = [int(x) for x in info]
    if not v[0]:
        return dict(zip(("mfma", "splits", "rows_per_item", "row_groups", "split_blocks"), v[:5]))
    # bf16: one persistent launch per row class (requests by Hq/Hkv * n_i)
    keys = ("workgroups", "rows_per_group", "row_groups", "units_per_workgroup")
    classes = [dict(zip(keys, v[1:5]), rows_lo=0, rows_hi=v[10])]
    if v[5] > 1:
        classes.append(dict(zip(keys, v[6:10]), rows_lo=v[10] + 1, rows_hi=2 ** 31 - 1))
    return dict(mfma=1, classes=classes, **classes[0])


def verify_attention(q, k_cache, v_cache, block_tables, seq_lens, q_start, *, max_q_len: int,
                     max_seq_len: int, sliding_window: int = 0, scale: float = 0.0,
                     kv_split_blocks: int = 0, sinks=None, out=None, workspace=None,
                     stream=None, check=None):
    """Attention of every packed query row against its request's paged KV cache.

    q [T, Hq, D]; k_cache [NB, Hkv, D/x, 16, x]; v_cache [NB, Hkv, D, 16] (bf16 or
    fp32, x = 16 bytes / element); block_tables [B, MB], seq_lens [B], q_start
    [B+1] int32 on the device.  max_q_len / max_seq_len are host upper bounds of
    n_i = q_start[i+1]-q_start[i] and S_i = seq_lens[i].  sinks: optional [Hq]
    float32 device tensor of per-head sink logits.  Returns `out`.  check:
    validate the descriptor on the device first (check_batch; raises
    BatchError, waits for the stream).
    """
    return _attention_call("verify_attention", q, None, k_cache, v_cache, block_tables, seq_lens, q_start,
                           max_q_len, max_seq_len, sliding_window, scale, kv_split_blocks, sinks, out,
                           workspace, stream, check)


def _attention_call(where, q, new, k_cache, v_cache, block_tables, seq_lens, q_start, max_q_len,
                    max_seq_len, sliding_window, scale, kv_split_blocks, sinks, out, workspace, stream,
                    check):
    """verify_attention, and with new = (k_new, v_new) verify_attention_append."""
    import torch
    if q.dim() != 3:
        raise ValueError("q must be [T, Hq, D], got %s" % (tuple(q.shape),))
    T, Hq, D = q.shape
    dtype, dev = q.dtype, q.device
    idx = dev.index if dev.type == "cuda" else -1
    p_q = _arg(q, "q", None, dtype, idx, dev)
    layer, params = _layer_args(Hq, D, dtype, q.element_size(), idx, dev, k_cache, v_cache, block_tables,
                                seq_lens, q_start)
    p_sinks = None if sinks is None else _arg(sinks, "sinks", (Hq,), torch.float32, idx, dev)
    p_out = None if out is None else _arg(out, "out", (T, Hq, D), dtype, idx, dev)
    p_ws, ws_have = _workspace_arg(workspace, idx, dev)
    p_new = []
    if new is not None:
        shape = (T, k_cache.shape[1], D)
        p_new = [_arg(new[0], "k_new", shape, dtype, idx, dev), _arg(new[1], "v_new", shape, dtype, idx, dev)]
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, where, q_start=q_start, total_q=T, max_q_len=max_q_len, seq_lens=seq_lens,
                 block_tables=block_tables, num_blocks=k_cache.shape[0], max_seq_len=max_seq_len,
                 sliding_window=sliding_window, stream=stream)
    params.sliding_window = int(sliding_window)
    params.scale = float(scale)
    params.kv_split_blocks = int(kv_split_blocks)
    if out is None:
        out = torch.empty_like(q)
        p_out = out.data_ptr()
    size = dict(max_q_len=max_q_len, max_seq_len=max_seq_len, sliding_window=sliding_window, scale=scale,
                kv_split_blocks=kv_split_blocks)
    if workspace is None:
        ws_have = attention_workspace_size(q, k_cache, block_tables, **size)
        if ws_have > 0:
            workspace = torch.empty(ws_have, dtype=torch.uint8, device=dev)
            p_ws = workspace.data_ptr()
    if idx < 0:
        _dev_ptr(q, "q")
    lib = library()
    call = lib.verify_attention if new is None else lib.verify_attention_append
    rc = call(ctypes.byref(params), T, int(max_q_len), int(max_seq_len), p_q, *p_new, *layer, p_sinks, p_out,
              p_ws, ws_have, _stream_ptr(stream, dev))
    if rc != OK:
        attention_workspace_size(q, k_cache, block_tables, **size)  # what it refuses is its error
        _check(rc, where)
    return out


def verify_attention_append(q, k_new, v_new, k_cache, v_cache, block_tables, seq_lens, q_start, *,
                            max_q_len: int, max_seq_len: int, sliding_window: int = 0,
                            scale: float = 0.0, kv_split_blocks: int = 0, sinks=None, out=None,
                            workspace=None, stream=None, check=None):
    """verify_kv_append and verify_attention in one launch sequence: the new
    tokens' K/V (k_new, v_new [T, Hkv, D], the cache's dtype) are stored into
    k_cache / v_cache in place while the attention reads them from k_new /
    v_new.  Same arguments and result as verify_attention; returns `out`."""
    return _attention_call("verify_attention_append", q, (k_new, v_new), k_cache, v_cache, block_tables,
                           seq_lens, q_start, max_q_len, max_seq_len, sliding_window, scale, kv_split_blocks,
                           sinks, out, workspace, stream, check)


def accept_workspace_size(num_seqs: int, total_q: int, vocab: int, dtype_code: int) -> int:
    n = ctypes.c_size_t(0)
    _check(library().verify_accept_workspace_size(int(num_seqs), int(total_q), int(vocab),
                                                  int(dtype_code), ctypes.byref(n)),
           "verify_accept_workspace_size")
    return int(n.value)


def _accept_outputs(T, q_start, argmax_out, accept_len, num_emitted, emitted, idx, dev):
    """Batch size, then the acceptance outputs (allocated where not given) and
    the addresses of q_start and of them."""
    import torch
    i32 = torch.int32
    if q_start.dim() != 1 or q_start.shape[0] < 1:
        raise ValueError("q_start must be [B + 1], got %s" % (tuple(q_start.shape),))
    B = q_start.shape[0] - 1
    p_qs = _arg(q_start, "q_start", None, i32, idx, dev)
    outs, ptrs = [], []
    for name, t, n in (("argmax_out", argmax_out, T), ("accept_len", accept_len, B),
                       ("num_emitted", num_emitted, B), ("emitted", emitted, T)):
        if t is None:
            t = torch.empty(n, dtype=i32, device=dev)
            ptrs.append(t.data_ptr())
        else:
            ptrs.append(_arg(t, name, (n,), i32, idx, dev))
        outs.append(t)
    return B, p_qs, outs, ptrs


def _accept_call(where, logits, tokens, q_start, outs, workspace, stream, check, draw=(), noalloc=False):
    """verify_accept, verify_accept_noalloc (noalloc) and verify_accept_sampled
    (draw = (temperature, seed, offset)); outs = (argmax or draw, accept_len,
    num_emitted, emitted), None where they are to be allocated."""
    import torch
    i32 = torch.int32
    if logits.dim() != 2:
        raise ValueError("logits must be [T, V], got %s" % (tuple(logits.shape),))
    T, V = logits.shape
    dev = logits.device
    idx = dev.index if dev.type == "cuda" else -1
    p_logits = _arg(logits, "logits", None, logits.dtype, idx, dev)
    B, p_qs, outs, (p_am, p_acc, p_num, p_em) = _accept_outputs(T, q_start, *outs, idx, dev)
    p_ws, ws_have = _workspace_arg(workspace, idx, dev)
    code = _dtype_code(logits)
    if workspace is None and not noalloc:
        ws_have = accept_workspace_size(B, T, V, code)
        if ws_have > 0:
            workspace = torch.empty(ws_have, dtype=torch.uint8, device=dev)
            p_ws = workspace.data_ptr()
    p_tok = _arg(tokens, "tokens", (T,), i32, idx, dev)
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, where, q_start=q_start, total_q=T, stream=stream)
    if idx < 0:
        _dev_ptr(logits, "logits")
    ws = () if noalloc else (p_ws, ws_have)
    rc = getattr(library(), where)(B, T, V, V, code, p_logits, p_tok, p_qs, *draw, p_am, p_acc, p_num, p_em, *ws,
                                   _stream_ptr(stream, dev))
    if rc != OK:
        if not noalloc:
            accept_workspace_size(B, T, V, code)  # what it refuses is its error
        _check(rc, where)
    return outs[1], outs[2], outs[3], outs[0]


def verify_accept(logits, tokens, q_start, *, argmax_out=None, accept_len=None, num_emitted=None,
                  emitted=None, workspace=None, stream=None, check=None):
    """Vocabulary argmax of every row and greedy acceptance of the drafts.

    logits [T, V] (bf16 or fp32), tokens [T] and q_start [B+1] int32 on the
    device.  Returns (accept_len [B], num_emitted [B], emitted [T], argmax [T]).
    check: validate q_start on the device first (check_batch).
    """
    return _accept_call("verify_accept", logits, tokens, q_start, (argmax_out, accept_len, num_emitted, emitted),
                        workspace, stream, check)


def verify_accept_noalloc(logits, tokens, q_start, *, argmax_out=None, accept_len=None,
                          num_emitted=None, emitted=None, stream=None, check=None):
    """verify_accept without a workspace: the library's per-GPU scratch array
    holds the partial maxima (for callers that cannot allocate; calls that
    overlap on one GPU race).  Outputs not passed in are allocated here, by
    torch, before the call; the C call allocates nothing.  Returns
    (accept_len [B], num_emitted [B], emitted [T], argmax [T])."""
    return _accept_call("verify_accept_noalloc", logits, tokens, q_start,
                        (argmax_out, accept_len, num_emitted, emitted), None, stream, check, noalloc=True)


def verify_accept_sampled(logits, tokens, q_start, *, temperature: float, seed: int, offset: int = 0,
                          sampled_out=None, accept_len=None, num_emitted=None, emitted=None,
                          workspace=None, stream=None, check=None):
    """Stochastic verification at temperature T > 0: every row draws
    y ~ softmax(logits / T) (Gumbel-max with Philox4x32-10 noise keyed by
    `seed`, counter (v / 4, row, offset, 0)) and a request accepts its drafts
    up to the first one that differs from its row's draw.

    Same layouts as verify_accept.  Returns (accept_len [B], num_emitted [B],
    emitted [T], sampled [T]).
    """
    if not 0 <= int(seed) < (1 << 64) or not 0 <= int(offset) < (1 << 32):
        raise ValueError("seed must fit 64 bits and offset 32 bits, unsigned")
    return _accept_call("verify_accept_sampled", logits, tokens, q_start,
                        (sampled_out, accept_len, num_emitted, emitted), workspace, stream, check,
                        draw=(float(temperature), int(seed), int(offset)))


def lmhead_accept_workspace_size(num_seqs: int, total_q: int, hidden_size: int, vocab: int,
                                 dtype_code: int = BF16) -> int:
    n = ctypes.c_size_t(0)
    _check(library().verify_lmhead_accept_workspace_size(int(num_seqs), int(total_q), int(hidden_size),
                                                         int(vocab), int(dtype_code), ctypes.byref(n)),
           "verify_lmhead_accept_workspace_size")
    return int(n.value)


def verify_lmhead_accept(hidden, weight, tokens, q_start, *, argmax_out=None, accept_len=None,
                         num_emitted=None, emitted=None, workspace=None, stream=None, check=None):
    """LM head fused with greedy acceptance: logits <hidden[r], weight[v]> are
    reduced to each row's argmax inside the kernel (never stored), then the
    drafts are accepted as in verify_accept.

    hidden [T, H] and weight [V, H] bf16, tokens [T] and q_start [B+1] int32,
    all on the device.  Returns (accept_len [B], num_emitted [B], emitted [T],
    argmax [T]).
    """
    import torch
    i32 = torch.int32
    if hidden.dim() != 2 or weight.dim() != 2:
        raise ValueError("hidden must be [T, H] and weight [V, H]")
    T, H = hidden.shape
    V, H2 = weight.shape
    if H != H2:
        raise ValueError("hidden sizes differ: %d vs %d" % (H, H2))
    dev, dtype = hidden.device, hidden.dtype
    idx = dev.index if dev.type == "cuda" else -1
    p_h = _arg(hidden, "hidden", None, dtype, idx, dev)
    p_w = _arg(weight, "weight", None, dtype, idx, dev)
    p_tok = _arg(tokens, "tokens", (T,), i32, idx, dev)
    B, p_qs, outs, (p_am, p_acc, p_num, p_em) = _accept_outputs(T, q_start, argmax_out, accept_len, num_emitted,
                                                                emitted, idx, dev)
    p_ws, ws_have = _workspace_arg(workspace, idx, dev)
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, "verify_lmhead_accept", q_start=q_start, total_q=T, stream=stream)
    code = _dtype_code(hidden)
    if workspace is None:
        ws_have = lmhead_accept_workspace_size(B, T, H, V, code)
        if ws_have > 0:
            workspace = torch.empty(ws_have, dtype=torch.uint8, device=dev)
            p_ws = workspace.data_ptr()
    if idx < 0:
        _dev_ptr(hidden, "hidden")
    rc = library().verify_lmhead_accept(B, T, H, V, code, p_h, p_w, p_tok, p_qs, p_am, p_acc, p_num, p_em, p_ws,
                                        ws_have, _stream_ptr(stream, dev))
    if rc != OK:
        lmhead_accept_workspace_size(B, T, H, V, code)  # what it refuses is its error
        _check(rc, "verify_lmhead_accept")
    return outs[1], outs[2], outs[3], outs[0]


def verify_budget(cand_start, cand_len, cand_tokens, last_token, *, alpha: float, g_min: float,
                  ctx_len=None, out=None, stream=None):
    """Redundancy-aware draft lengths (Sec. 4.2, Alg. 2) and the next verify
    step's descriptor.

    cand_start [B+1], cand_len [C], cand_tokens [C, max_len], last_token [B]
    and ctx_len [B] (optional) are int32 device tensors.  Returns a dict of
    device tensors: score (float64), agree, prefix_len, source, draft_len,
    q_start, tokens (capacity B * (max_len + 1); q_start[-1] entries used) and,
    with ctx_len, seq_lens.  ``out`` may hold preallocated tensors by name.
    """
    import torch
    if cand_start.dim() != 1 or cand_start.shape[0] < 1 or cand_tokens.dim() != 2:
        raise ValueError("cand_start must be [B + 1] and cand_tokens [C, max_len]")
    B = cand_start.shape[0] - 1
    C, max_len = cand_tokens.shape
    dev = cand_start.device
    idx = dev.index if dev.type == "cuda" else -1
    i32, f64 = torch.int32, torch.float64
    p_start = _arg(cand_start, "cand_start", None, i32, idx, dev)
    p_len = _arg(cand_len, "cand_len", (C,), i32, idx, dev)
    p_cand = _arg(cand_tokens, "cand_tokens", None, i32, idx, dev)
    p_last = _arg(last_token, "last_token", (B,), i32, idx, dev)
    p_ctx = None if ctx_len is None else _arg(ctx_len, "ctx_len", (B,), i32, idx, dev)
    o = dict(out or {})
    shapes = [("score", B, f64), ("agree", B, i32), ("prefix_len", B, i32), ("source", B, i32),
              ("draft_len", B, i32), ("q_start", B + 1, i32), ("tokens", B * (max_len + 1), i32)]
    if ctx_len is not None:
        shapes.append(("seq_lens", B, i32))
    ptrs = []
    for k, n, dt in shapes:
        if k not in o:
            o[k] = t = torch.empty(max(n, 1) if k == "tokens" else n, dtype=dt, device=dev)
            ptrs.append(t.data_ptr())
        elif k == "tokens":
            # the capacity is passed to the call, which checks it
            ptrs.append(_arg(o[k], k, None, dt, idx, dev))
            if o[k].dim() != 1:
                raise ValueError("tokens must be one-dimensional")
        else:
            ptrs.append(_arg(o[k], k, (n,), dt, idx, dev))
    if ctx_len is None:
        ptrs.append(_dev_ptr(o.get("seq_lens"), "seq_lens", i32))
    if idx < 0:
        _dev_ptr(cand_start, "cand_start")
    rc = library().verify_budget(B, C, max_len, p_start, p_len, p_cand, p_last, p_ctx, float(alpha), float(g_min),
                                 *ptrs[:7], o["tokens"].numel(), ptrs[7], _stream_ptr(stream, dev))
    _check(rc, "verify_budget")
    return o


def verify_kv_append(k_new, v_new, k_cache, v_cache, block_tables, seq_lens, q_start, *,
                     stream=None, check=None):
    """Write the new tokens' K/V ([T, Hkv, D], the cache's dtype) into their
    paged-cache slots (position S_i - n_i + j for row j of request i), in place.
    check: validate the descriptor and the new tokens' block ids on the device
    first (check_batch with a one-key window: only those blocks)."""
    if k_new.dim() != 3:
        raise ValueError("k_new must be [T, Hkv, D], got %s" % (tuple(k_new.shape),))
    _expect(v_new, "v_new", tuple(k_new.shape), k_new.dtype, k_new.device)
    if q_start.dim() != 1 or q_start.shape[0] < 1:
        raise ValueError("q_start must be [B + 1], got %s" % (tuple(q_start.shape),))
    T, hkv, D = k_new.shape
    dtype, dev = k_new.dtype, k_new.device
    idx = dev.index if dev.type == "cuda" else -1
    p_k, p_v = _arg(k_new, "k_new", None, dtype, idx, dev), _arg(v_new, "v_new", None, dtype, idx, dev)
    (p_kc, p_vc, *desc), params = _layer_args(hkv, D, dtype, k_new.element_size(), idx, dev, k_cache, v_cache,
                                              block_tables, seq_lens, q_start)
    if k_cache.shape[1] != hkv:
        raise ValueError("k_new has %d KV heads, the cache %d" % (hkv, k_cache.shape[1]))
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, "verify_kv_append", q_start=q_start, total_q=T, seq_lens=seq_lens,
                 block_tables=block_tables, num_blocks=k_cache.shape[0],
                 max_seq_len=16 * block_tables.shape[1], sliding_window=1, stream=stream)
    if idx < 0:
        _dev_ptr(k_new, "k_new")
    rc = library().verify_kv_append(ctypes.byref(params), T, p_k, p_v, *desc, p_kc, p_vc, _stream_ptr(stream, dev))
    _check(rc, "verify_kv_append")


def _scratch(shape, dtype, dev, stream):
    """A tensor that a call on `stream` (None: the current one) uses, from that
    stream's memory: its last use there is over before this one begins."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


_current_device = None


def _launch(where, idx, *args):
    """The library's call `where` with the tensors' device current, as a launch on
    one of its streams needs."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    call = getattr(_lib or library(), where)
    if _current_device() == idx:
        rc = call(*args)
    else:
        import torch
        with torch.cuda.device(idx):
            rc = call(*args)
    if rc != OK:
        _check(rc, where)


def _rows_arg(t, name, heads, D, dtype, idx, device, T):
    """Address and row stride of packed rows [T, heads, D]: contiguous, or a slice
    of wider rows (heads and dims adjacent, any row stride that holds them)."""
    shape = (T, heads, D)
    if not (t is not None and t.dtype is dtype and t.get_device() == idx >= 0 and t.shape == shape):
        _expect(t, name, shape, dtype, device)
    if t.is_contiguous():
        return t.data_ptr(), heads * D
    st = t.stride()
    if T <= 1:
        st = (heads * D,) + st[1:]  # one row has no stride
    if (st[2] != 1 and D > 1) or (st[1] != D and heads > 1) or st[0] < heads * D:
        raise ValueError("%s must be rows of %d x %d adjacent elements, got strides %s" % (name, heads, D, tuple(st)))
    return t.data_ptr(), st[0]


_rotary_params = {}


def _rotary_args(q, T, D, positions, inv_freq, axes, interleaved, scale, idx, dev):
    """RotaryParams of a call, and the addresses of positions and inv_freq."""
    import torch
    if inv_freq.dim() != 1:
        raise ValueError("inv_freq must be [rotary_dim / 2], got %s" % (tuple(inv_freq.shape),))
    F = inv_freq.numel()
    one = positions.dim() == 1
    num_axes = 1 if one else positions.shape[0]
    if num_axes != 1 if axes is None else len(axes) != F:
        raise ValueError("axes must name the axis of each of the %d frequencies" % F)
    p_pos = _arg(positions, "positions", (T,) if one else (num_axes, T), torch.int32, idx, dev)
    p_freq = _arg(inv_freq, "inv_freq", None, torch.float64, idx, dev)
    try:
        # of the usual 64 small numbers a string of bytes is made, hashed and compared in
        # half of a tuple's time; of others than a list bytes() may take the memory (arrays)
        # or a length (a tensor of one number)
        turned = None if axes is None else bytes(axes if type(axes) in (list, tuple) else [int(x) for x in axes])
    except (TypeError, ValueError):
        turned = tuple(int(x) for x in axes)
    key = (D, F, num_axes, bool(interleaved), float(scale), q.dtype, turned)
    params = _rotary_params.get(key)
    if params is None:
        axes = (0,) * F if axes is None else axes
        if not (2 <= 2 * F <= D and all(0 <= int(x) < num_axes for x in axes)):
            raise ValueError("rotary_dim %d of head dim %d, axes %s of %d" % (2 * F, D, sorted(set(axes)), num_axes))
        params = RotaryParams(D, 2 * F, num_axes, int(bool(interleaved)), float(scale), _dtype_code(q))
        for f, x in enumerate(axes):
            if f < len(params.axis):
                params.axis[f] = int(x)
        if len(_rotary_params) > 64:
            _rotary_params.clear()
        _rotary_params[key] = params
    return params, p_pos, p_freq


def verify_rotary(q, k, positions, inv_freq, *, axes=None, interleaved: bool = False, scale: float = 0.0,
                  q_out=None, k_out=None, stream=None):
    """Queries and keys rotated to their rows' positions.

    q [T, Hq, D] and k [T, Hkv, D] or None (bf16 or fp32, D 64 or 128), contiguous
    or slices of wider rows; positions [A, T] (or [T]) int32; inv_freq [R / 2]
    float64, radians per position; axes: the axis (0 .. A-1) of each of the R / 2
    frequencies, needed with more than one.  A pair is dims (f, f + R / 2), or
    (2f, 2f + 1) if interleaved; dims from R on are copied.  scale: a factor of the
    rotated dims (0: 1).  q_out and k_out may be q and k.  Returns (q_out, k_out)."""
    return _rotary_call("verify_rotary", None, q, k, positions, inv_freq, axes, interleaved, scale, q_out, k_out, stream)


def verify_norm_rotary(q, k, positions, inv_freq, *, q_weight=None, k_weight=None, eps: float = 1e-6, axes=None,
                       interleaved: bool = False, scale: float = 0.0, q_out=None, k_out=None, stream=None):
    """verify_rotary behind a norm of each head: x * weight / sqrt(mean(x^2) + eps) over
    the head's D dims, with q_weight and k_weight [D] float32 (None: ones).  Norm and
    rotation are rounded once.  Other arguments and the result as for verify_rotary."""
    return _rotary_call("verify_norm_rotary", (q_weight, k_weight, eps), q, k, positions, inv_freq, axes, interleaved,
                        scale, q_out, k_out, stream)


def _norm_args(norm, D, idx, dev):
    """The norm's arguments of a call: none for a call without one."""
    if norm is None:
        return ()
    import torch
    q_weight, k_weight, eps = norm
    return (None if q_weight is None else _arg(q_weight, "q_weight", (D,), torch.float32, idx, dev),
            None if k_weight is None else _arg(k_weight, "k_weight", (D,), torch.float32, idx, dev), float(eps))


def _rotary_call(where, norm, q, k, positions, inv_freq, axes, interleaved, scale, q_out, k_out, stream):
    if q.dim() != 3 or k is not None and k.dim() != 3:
        raise ValueError("q must be [T, Hq, D] and k [T, Hkv, D]")
    T, Hq, D = q.shape
    dtype, dev, idx = q.dtype, q.device, q.get_device()
    Hkv = 0 if k is None else k.shape[1]
    p_q, s_q = _rows_arg(q, "q", Hq, D, dtype, idx, dev, T)
    p_k, s_k = (None, 0) if k is None else _rows_arg(k, "k", Hkv, D, dtype, idx, dev, T)
    params, p_pos, p_freq = _rotary_args(q, T, D, positions, inv_freq, axes, interleaved, scale, idx, dev)
    norm = _norm_args(norm, D, idx, dev)
    if q_out is None:
        q_out = _scratch((T, Hq, D), dtype, dev, stream)
    if k_out is None and k is not None:
        k_out = _scratch((T, Hkv, D), dtype, dev, stream)
    p_qo, s_qo = _rows_arg(q_out, "q_out", Hq, D, dtype, idx, dev, T)
    p_ko, s_ko = (None, 0) if k is None else _rows_arg(k_out, "k_out", Hkv, D, dtype, idx, dev, T)
    if idx < 0:
        _dev_ptr(q, "q")
    _launch(where, idx, ctypes.byref(params), T, Hq, Hkv, p_q, s_q, p_k, s_k, *norm, p_pos, p_freq, p_qo, s_qo,
            p_ko, s_ko, _stream_ptr(stream, dev))
    return q_out, k_out


def verify_rotary_append(q, k_new, v_new, positions, inv_freq, k_cache, v_cache, block_tables, seq_lens, q_start, *,
                         axes=None, interleaved: bool = False, scale: float = 0.0, q_out=None, stream=None,
                         check=None):
    """verify_rotary with the rotated keys and the values written into their
    paged-cache slots in the same launch (as verify_kv_append writes them).  q [T,
    Hq, D], k_new and v_new [T, Hkv, D], contiguous or slices of wider rows.  check:
    as for verify_kv_append.  Returns q_out."""
    return _rotary_append_call("verify_rotary_append", None, q, k_new, v_new, positions, inv_freq, k_cache, v_cache,
                               block_tables, seq_lens, q_start, axes, interleaved, scale, q_out, stream, check)


def verify_norm_rotary_append(q, k_new, v_new, positions, inv_freq, k_cache, v_cache, block_tables, seq_lens, q_start,
                              *, q_weight=None, k_weight=None, eps: float = 1e-6, axes=None,
                              interleaved: bool = False, scale: float = 0.0, q_out=None, stream=None, check=None):
    """verify_rotary_append behind a norm of each head's query and key (see
    verify_norm_rotary; the values are stored as they are).  Returns q_out."""
    return _rotary_append_call("verify_norm_rotary_append", (q_weight, k_weight, eps), q, k_new, v_new, positions,
                               inv_freq, k_cache, v_cache, block_tables, seq_lens, q_start, axes, interleaved, scale,
                               q_out, stream, check)


def _rotary_append_call(where, norm, q, k_new, v_new, positions, inv_freq, k_cache, v_cache, block_tables, seq_lens,
                        q_start, axes, interleaved, scale, q_out, stream, check):
    if q.dim() != 3 or k_new.dim() != 3 or v_new.dim() != 3:
        raise ValueError("q must be [T, Hq, D], k_new and v_new [T, Hkv, D]")
    T, Hq, D = q.shape
    dtype, dev, idx = q.dtype, q.device, q.get_device()
    p_q, s_q = _rows_arg(q, "q", Hq, D, dtype, idx, dev, T)
    (p_kc, p_vc, *desc), attn = _layer_args(Hq, D, dtype, q.element_size(), idx, dev, k_cache, v_cache, block_tables,
                                            seq_lens, q_start, own=False)
    Hkv = attn.num_kv_heads
    p_k, s_k = _rows_arg(k_new, "k_new", Hkv, D, dtype, idx, dev, T)
    p_v, s_v = _rows_arg(v_new, "v_new", Hkv, D, dtype, idx, dev, T)
    params, p_pos, p_freq = _rotary_args(q, T, D, positions, inv_freq, axes, interleaved, scale, idx, dev)
    norm = _norm_args(norm, D, idx, dev)
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, where, q_start=q_start, total_q=T, seq_lens=seq_lens,
                 block_tables=block_tables, num_blocks=k_cache.shape[0],
                 max_seq_len=16 * block_tables.shape[1], sliding_window=1, stream=stream)
    if q_out is None:
        q_out = _scratch((T, Hq, D), dtype, dev, stream)
    p_qo, s_qo = _rows_arg(q_out, "q_out", Hq, D, dtype, idx, dev, T)
    if idx < 0:
        _dev_ptr(q, "q")
    _launch(where, idx, ctypes.byref(attn), ctypes.byref(params), T, p_q, s_q, p_k, s_k, p_v, s_v, *norm, p_pos,
            p_freq, *desc, p_qo, s_qo, p_kc, p_vc, _stream_ptr(stream, dev))
    return q_out


def _row_matrix(t, name, shape, dtype, idx, device):
    """Address and row stride of a matrix whose rows are contiguous."""
    if not (t is not None and t.dtype is dtype and t.get_device() == idx >= 0 and t.shape == shape):
        _expect(t, name, shape, dtype, device)
    if t.is_contiguous():
        return t.data_ptr(), shape[1]
    rows, stride = shape[0], t.stride()
    if shape[1] > 1 and stride[1] != 1 or rows > 1 and stride[0] < shape[1]:
        raise ValueError("%s must have rows of %d adjacent elements, got strides %s" % (name, shape[1], tuple(stride)))
    return t.data_ptr(), stride[0] if rows > 1 else shape[1]


def _token_state(counts, seen, slots, vocab, B, idx, dev, i32):
    """Addresses of a state of token counts and bits and of the requests' slots in it,
    and its number of slots."""
    if counts.dim() != 2:
        raise ValueError("counts must be [slots, V], got %s" % (tuple(counts.shape),))
    n = counts.shape[0]
    if slots is None and n < B:
        raise ValueError("%d requests have %d slots: name them in slots" % (B, n))
    return (_arg(counts, "counts", (n, vocab), i32, idx, dev),
            _arg(seen, "seen", (n, 2, (vocab + 31) // 32), i32, idx, dev),
            None if slots is None else _arg(slots, "slots", (B,), i32, idx, dev), n)


def verify_adjust_logits(logits, tokens, q_start, *, counts=None, seen=None, slots=None, repetition=None,
                         frequency=None, presence=None, bias_start=None, bias_tokens=None, bias_values=None,
                         mask=None, mask_rows=None, out=None, stream=None, check=None):
    """Penalties, biases and grammar masks, before verify_accept or verify_accept_sampled
    reads the logits.

    logits [T, V] (bf16 or fp32, rows may be strided), tokens [T] and q_start [B + 1] as
    for verify_accept: row j of a request is scored behind its drafts 1 .. j, which
    count.  repetition, frequency, presence [B] float32 or None; with any of them counts
    [slots, V] int32 and seen [slots, 2, ceil(V / 32)] int32 are the state that
    verify_count_tokens keeps (zeros for a new request), slots [B] int32 the requests'
    rows in it (None: 0 .. B-1).  bias_start [B + 1], bias_tokens and bias_values: each
    request's list of biased tokens.  mask [M, ceil(V / 32)] int32 bits (token v: bit
    v % 32 of word v // 32) of the tokens that may follow, mask_rows [T] each row's mask
    (-1: all may).  out: None for a new tensor; logits to change them in place.  Returns
    out."""
    import torch
    i32, f32 = torch.int32, torch.float32
    if logits.dim() != 2:
        raise ValueError("logits must be [T, V], got %s" % (tuple(logits.shape),))
    T, V = logits.shape
    dev, dtype, idx = logits.device, logits.dtype, logits.get_device()
    if q_start.dim() != 1 or q_start.numel() < 1:
        raise ValueError("q_start must be [B + 1], got %s" % (tuple(q_start.shape),))
    B = q_start.numel() - 1
    code = _dtype_code(logits)
    p_logits, stride = _row_matrix(logits, "logits", (T, V), dtype, idx, dev)
    p_qs = _arg(q_start, "q_start", None, i32, idx, dev)
    p_tok = None if tokens is None else _arg(tokens, "tokens", (T,), i32, idx, dev)
    state, bias, masks = (None,) * 6 + (0,), (None,) * 3 + (0,), (0, None, None)
    if repetition is not None or frequency is not None or presence is not None:
        if counts is None or seen is None or tokens is None:
            raise ValueError("a penalty needs counts, seen and tokens")
        state = (None if repetition is None else _arg(repetition, "repetition", (B,), f32, idx, dev),
                 None if frequency is None else _arg(frequency, "frequency", (B,), f32, idx, dev),
                 None if presence is None else _arg(presence, "presence", (B,), f32, idx, dev),
                 *_token_state(counts, seen, slots, V, B, idx, dev, i32))
    if bias_start is not None:
        if bias_tokens is None or bias_values is None or bias_tokens.dim() != 1:
            raise ValueError("bias_start needs bias_tokens and bias_values of one dim")
        m = bias_tokens.numel()
        bias = (_arg(bias_start, "bias_start", (B + 1,), i32, idx, dev),
                _arg(bias_tokens, "bias_tokens", None, i32, idx, dev),
                _arg(bias_values, "bias_values", (m,), f32, idx, dev), m)
    elif bias_tokens is not None or bias_values is not None:
        raise ValueError("bias_tokens and bias_values need bias_start")
    if mask_rows is not None:
        if mask is None or mask.dim() != 2:
            raise ValueError("mask_rows needs mask [M, ceil(V / 32)]")
        masks = (mask.shape[0], _arg(mask, "mask", (mask.shape[0], (V + 31) // 32), i32, idx, dev),
                 _arg(mask_rows, "mask_rows", (T,), i32, idx, dev))
    elif mask is not None:
        raise ValueError("mask needs mask_rows")
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, "verify_adjust_logits", q_start=q_start, total_q=T, stream=stream)
    if out is None:
        out = _scratch((T, V), dtype, dev, stream)
    p_out, out_stride = _row_matrix(out, "out", (T, V), dtype, idx, dev)
    if idx < 0:
        _dev_ptr(logits, "logits")
    _launch("verify_adjust_logits", idx, B, T, V, stride, code, p_logits, p_tok, p_qs,
            ctypes.byref(AdjustParams(*state, *bias, *masks)), p_out, out_stride, _stream_ptr(stream, dev))
    return out


def verify_count_tokens(counts, seen, tokens, token_start, *, num_tokens=None, slots=None, prompt: bool = False,
                        stream=None):
    """Enters tokens into the state that verify_adjust_logits reads, in place.

    counts [slots, V] and seen [slots, 2, ceil(V / 32)] int32 (zeros for a new request).
    Request i's tokens are the first num_tokens[i] (None: all) of tokens[token_start[i]
    : token_start[i + 1]]: after an acceptance tokens = emitted, token_start = q_start
    and num_tokens = num_emitted.  prompt: they belong to the request's prompt, which
    only the repetition penalty regards.  Tokens outside the vocabulary are passed
    over.  slots [B] int32: the requests' rows of the state (None: 0 .. B-1)."""
    import torch
    i32 = torch.int32
    if token_start.dim() != 1 or token_start.numel() < 1:
        raise ValueError("token_start must be [B + 1], got %s" % (tuple(token_start.shape),))
    if tokens.dim() != 1:
        raise ValueError("tokens must be packed in one dim, got %s" % (tuple(tokens.shape),))
    B, V, dev, idx = token_start.numel() - 1, counts.shape[-1], counts.device, counts.get_device()
    p_counts, p_seen, p_slots, n = _token_state(counts, seen, slots, V, B, idx, dev, i32)
    p_tok = _arg(tokens, "tokens", None, i32, idx, dev)
    p_start = _arg(token_start, "token_start", None, i32, idx, dev)
    p_num = None if num_tokens is None else _arg(num_tokens, "num_tokens", (B,), i32, idx, dev)
    if idx < 0:
        _dev_ptr(counts, "counts")
    _launch("verify_count_tokens", idx, B, tokens.numel(), V, n, p_tok, p_start, p_num, p_slots,
            int(bool(prompt)), p_counts, p_seen, _stream_ptr(stream, dev))


def _workspace_size(where, params, *bounds):
    """The size query `where`, in bytes."""
    n = ctypes.c_size_t(0)
    _check(getattr(library(), where)(ctypes.byref(params), *bounds, ctypes.byref(n)), where)
    return int(n.value)


def attention_shared_workspace_size(q, k_cache, block_tables, *, num_groups: int, max_q_len: int, max_seq_len: int,
                                    max_prefix_len: int) -> int:
    return _workspace_size("verify_attention_shared_workspace_size", _attn_params(q, k_cache, block_tables, 0, 0.0, 0),
                           q.shape[0], int(max_q_len), int(max_seq_len), int(num_groups), int(max_prefix_len))


def verify_attention_shared(q, k_cache, v_cache, block_tables, seq_lens, q_start, group_start, prefix_lens, *,
                            max_q_len: int, max_seq_len: int, max_prefix_len: int, scale: float = 0.0, sinks=None,
                            out=None, workspace=None, stream=None, check=None):
    """verify_attention of a batch in which groups of requests begin with the same cached
    tokens: the keys of a common prefix are read once for all rows of its group.

    group_start [G + 1] int32: requests group_start[k] .. group_start[k + 1] - 1 form
    group k; prefix_lens [G] int32: their first prefix_lens[k] // 16 block table entries
    are the same; max_prefix_len bounds them.  k_cache, v_cache and workspace are 16-byte
    aligned.  check also refuses groups that fail check_groups.  Other arguments and the
    result as for verify_attention without a window."""
    import torch
    if q.dim() != 3:
        raise ValueError("q must be [T, Hq, D], got %s" % (tuple(q.shape),))
    if group_start.dim() != 1 or group_start.numel() < 1:
        raise ValueError("group_start must be [G + 1], got %s" % (tuple(group_start.shape),))
    T, Hq, D = q.shape
    dtype, dev, idx = q.dtype, q.device, q.get_device()
    G = group_start.numel() - 1
    p_q = _arg(q, "q", None, dtype, idx, dev)
    layer, params = _layer_args(Hq, D, dtype, q.element_size(), idx, dev, k_cache, v_cache, block_tables, seq_lens,
                                q_start, own=scale != 0.0)
    p_gs = _arg(group_start, "group_start", None, torch.int32, idx, dev)
    p_pl = _arg(prefix_lens, "prefix_lens", (G,), torch.int32, idx, dev)
    p_sinks = None if sinks is None else _arg(sinks, "sinks", (Hq,), torch.float32, idx, dev)
    p_ws, ws_have = _workspace_arg(workspace, idx, dev)
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, "verify_attention_shared", q_start=q_start, total_q=T, max_q_len=max_q_len, seq_lens=seq_lens,
                 block_tables=block_tables, num_blocks=k_cache.shape[0], max_seq_len=max_seq_len, stream=stream)
        bad, first = check_groups(group_start, prefix_lens, seq_lens, block_tables, max_prefix_len=max_prefix_len,
                                  max_seq_len=max_seq_len, stream=stream)
        if any(bad.values()):
            raise BatchError("verify_attention_shared", bad, first, "group")
    if scale != 0.0:
        params.scale = scale
    bounds = T, int(max_q_len), int(max_seq_len), G, int(max_prefix_len)
    if out is None:
        out = _scratch((T, Hq, D), dtype, dev, stream)
    p_out = _arg(out, "out", (T, Hq, D), dtype, idx, dev)
    if workspace is None:
        ws_have = _workspace_size("verify_attention_shared_workspace_size", params, *bounds)
        if ws_have > 0:
            workspace = _scratch(ws_have, torch.uint8, dev, stream)
            p_ws = workspace.data_ptr()
    if idx < 0:
        _dev_ptr(q, "q")
    _launch("verify_attention_shared", idx, ctypes.byref(params), *bounds, p_q, *layer, p_gs, p_pl, p_sinks, p_out,
            p_ws, ws_have, _stream_ptr(stream, dev))
    return out


def key_weights_workspace_size(q, k_cache, block_tables, *, max_q_len: int, max_seq_len: int) -> int:
    return _workspace_size("verify_key_weights_workspace_size", _attn_params(q, k_cache, block_tables, 0, 0.0, 0),
                           q.shape[0], int(max_q_len), int(max_seq_len))


def verify_key_weights(q, k_cache, key_weights, key_order, block_tables, seq_lens, q_start, *, max_q_len: int,
                       max_seq_len: int, num_rows=None, num_tokens=None, sinks=None, scale: float = 0.0,
                       decay: float = 1.0, workspace=None, stream=None, check=None):
    """Adds the attention weights of the step's rows to the cached keys' sums.

    key_weights [num_blocks, Hkv, 16] float32 and key_order [num_blocks, Hkv, 16]
    int32 are updated in place: a key held before the step gets decay * its sum plus
    its weight in the rows' softmaxes (summed over the rows and the query heads of
    its KV head), a new one that weight and the ordinal of its token.  num_rows [B]:
    only the first num_rows[i] rows of request i count (after an acceptance,
    num_emitted).  num_tokens [B]: the request's tokens so far with the new ones
    (None: seq_lens).  Other arguments as for verify_attention, after the append
    (check=True also refuses a request of more than max_q_len rows, which the call
    itself takes).  Returns key_weights."""
    import torch
    if q.dim() != 3:
        raise ValueError("q must be [T, Hq, D], got %s" % (tuple(q.shape),))
    T, Hq, D = q.shape
    dtype, dev, idx = q.dtype, q.device, q.get_device()
    p_q = _arg(q, "q", None, dtype, idx, dev)
    p_kc, params = _key_cache_arg(k_cache, Hq, D, dtype, q.element_size(), idx, dev)
    nb, hkv = k_cache.shape[0], k_cache.shape[1]
    p_bt, p_sl, B = _table_args(params, block_tables, seq_lens, idx, dev)
    p_qs = _arg(q_start, "q_start", (B + 1,), torch.int32, idx, dev)
    p_w, p_o = _key_state(key_weights, key_order, nb, hkv, idx, dev)
    p_rows = None if num_rows is None else _arg(num_rows, "num_rows", (B,), torch.int32, idx, dev)
    p_tok = None if num_tokens is None else _arg(num_tokens, "num_tokens", (B,), torch.int32, idx, dev)
    p_sinks = None if sinks is None else _arg(sinks, "sinks", (Hq,), torch.float32, idx, dev)
    p_ws, ws_have = _workspace_arg(workspace, idx, dev)
    if check or check is None and CHECK_BY_DEFAULT:
        _checked(check, "verify_key_weights", q_start=q_start, total_q=T, max_q_len=max_q_len, seq_lens=seq_lens,
                 block_tables=block_tables, num_blocks=nb, max_seq_len=max_seq_len, stream=stream)
    params.scale = float(scale)
    if workspace is None:
        ws_have = _workspace_size("verify_key_weights_workspace_size", params, T, int(max_q_len), int(max_seq_len))
        if ws_have > 0:
            workspace = _scratch(ws_have, torch.uint8, dev, stream)
            p_ws = workspace.data_ptr()
    if idx < 0:
        _dev_ptr(q, "q")
    _launch("verify_key_weights", idx, ctypes.byref(params), T, int(max_q_len), int(max_seq_len), p_q, p_kc, p_bt,
            p_sl, p_qs, p_rows, p_tok, p_sinks, float(decay), p_w, p_o, p_ws, ws_have, _stream_ptr(stream, dev))
    return key_weights


def _key_cache_arg(k_cache, Hq, D, dtype, esize, idx, dev):
    """Address of a key cache, and its AttnParams (num_seqs and the table's width are
    _table_args')."""
    if k_cache.dim() != 5:
        raise ValueError("k_cache must be [num_blocks, Hkv, D/x, 16, x], got %s" % (tuple(k_cache.shape),))
    nb, hkv = k_cache.shape[0], k_cache.shape[1]
    x = 16 // esize
    p = _arg(k_cache, "k_cache", (nb, hkv, D // x, 16, x), dtype, idx, dev)
    return p, AttnParams(0, Hq, hkv, D, 16, 0, nb, 0, 0.0, _dtype_code(k_cache), 0)


def _table_args(params, block_tables, lens, idx, dev, name="seq_lens"):
    """Addresses of block_tables and of the requests' lengths, and their number."""
    import torch
    if block_tables.dim() != 2:
        raise ValueError("block_tables must be [B, max_blocks], got %s" % (tuple(block_tables.shape),))
    B, params.max_blocks_per_seq = block_tables.shape
    params.num_seqs = B
    return (_arg(block_tables, "block_tables", None, torch.int32, idx, dev),
            _arg(lens, name, (B,), torch.int32, idx, dev), B)


def _key_state(key_weights, key_order, nb, hkv, idx, dev):
    import torch
    return (None if key_weights is None else _arg(key_weights, "key_weights", (nb, hkv, 16), torch.float32, idx, dev),
            None if key_order is None else _arg(key_order, "key_order", (nb, hkv, 16), torch.int32, idx, dev))


def evict_plan_workspace_size(num_seqs: int, num_kv_heads: int, max_blocks: int, *, max_seq_len: int,
                              max_keys: int) -> int:
    params = AttnParams(int(num_seqs), int(num_kv_heads), int(num_kv_heads), 128, 16, int(max_blocks), 0, 0, 0.0, BF16, 0)
    return _workspace_size("verify_evict_plan_workspace_size", params, int(max_seq_len), int(max_keys))


def verify_evict_plan(key_weights, key_order, block_tables, seq_lens, *, max_keys: int, keep_first: int = 0,
                      keep_recent: int = 0, max_seq_len: int, num_tokens=None, source=None, new_lens=None,
                      workspace=None, stream=None):
    """The keys to keep of requests that hold more than max_keys: for every KV head
    the tokens of the first keep_first and the last keep_recent ordinals, then the
    keys of the largest key_weights (the lower slot among equals).

    key_weights and key_order (None: the slot is the ordinal) as for
    verify_key_weights; num_tokens [B] or None (seq_lens).  Returns (source [B, Hkv,
    max_keys] int32: the slot whose key slot d is to hold, -1 from the request's new
    length on; new_lens [B] int32: min(seq_lens, max_keys)).  Nothing is moved."""
    import torch
    i32 = torch.int32
    if key_weights.dim() != 3:
        raise ValueError("key_weights must be [num_blocks, Hkv, 16], got %s" % (tuple(key_weights.shape),))
    dev, idx = key_weights.device, key_weights.get_device()
    nb, hkv = key_weights.shape[:2]
    p_w, p_o = _key_state(key_weights, key_order, nb, hkv, idx, dev)
    # the plan depends neither on the head dim nor on the storage type
    params = AttnParams(0, hkv, hkv, 128, 16, 0, nb, 0, 0.0, BF16, 0)
    p_bt, p_sl, B = _table_args(params, block_tables, seq_lens, idx, dev)
    p_tok = None if num_tokens is None else _arg(num_tokens, "num_tokens", (B,), i32, idx, dev)
    max_keys = int(max_keys)
    if source is None:
        source = _scratch((B, hkv, max(max_keys, 0)), i32, dev, stream)
    if new_lens is None:
        new_lens = _scratch((B,), i32, dev, stream)
    p_src = _arg(source, "source", (B, hkv, max(max_keys, 0)), i32, idx, dev)
    p_new = _arg(new_lens, "new_lens", (B,), i32, idx, dev)
    p_ws, ws_have = _workspace_arg(workspace, idx, dev)
    if workspace is None:
        ws_have = _workspace_size("verify_evict_plan_workspace_size", params, int(max_seq_len), max_keys)
        if ws_have > 0:
            workspace = _scratch(ws_have, torch.uint8, dev, stream)
            p_ws = workspace.data_ptr()
    if idx < 0:
        _dev_ptr(key_weights, "key_weights")
    _launch("verify_evict_plan", idx, ctypes.byref(params), int(max_seq_len), max_keys, int(keep_first),
            int(keep_recent), p_w, p_o, p_bt, p_sl, p_tok, p_src, p_new, p_ws, ws_have, _stream_ptr(stream, dev))
    return source, new_lens


def verify_kv_compact(k_cache, v_cache, block_tables, source, new_lens, *, key_weights=None, key_order=None,
                      stream=None):
    """Moves the kept keys, in place: slot d of every request and KV head receives
    the key, value (and weight and ordinal) of slot source[i, g, d] for d <
    new_lens[i].  source and new_lens as verify_evict_plan returns them, or a plan of
    the caller's own in which no slot that is moved from is moved to."""
    import torch
    i32 = torch.int32
    if k_cache.dim() != 5 or source.dim() != 3:
        raise ValueError("k_cache must be [num_blocks, Hkv, D/x, 16, x] and source [B, Hkv, max_keys]")
    dtype, dev, idx = k_cache.dtype, k_cache.device, k_cache.get_device()
    nb, hkv = k_cache.shape[:2]
    D = k_cache.shape[2] * k_cache.shape[4]
    p_kc, params = _key_cache_arg(k_cache, hkv, D, dtype, k_cache.element_size(), idx, dev)
    p_vc = _arg(v_cache, "v_cache", (nb, hkv, D, 16), dtype, idx, dev)
    p_bt, p_new, B = _table_args(params, block_tables, new_lens, idx, dev, "new_lens")
    p_src = _arg(source, "source", (B, hkv, source.shape[2]), i32, idx, dev)
    p_w, p_o = _key_state(key_weights, key_order, nb, hkv, idx, dev)
    if idx < 0:
        _dev_ptr(k_cache, "k_cache")
    _launch("verify_kv_compact", idx, ctypes.byref(params), source.shape[2], p_bt, p_src, p_new, p_kc, p_vc, p_w,
            p_o, _stream_ptr(stream, dev))
