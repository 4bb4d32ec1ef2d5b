"""The calls that keep a request's paged KV cache within a bound, as measured cases.

A serving engine that bounds its caches makes these calls around the attention of
every layer: the new tokens' queries and keys are rotated to their positions (given
explicitly, on one axis or on several, since an evicted cache's slots say nothing of
positions) and the keys and values appended; each cached key's attention weight is
accumulated; the keys to keep are chosen; the kept ones move into the slots of those
that leave.  A case is one such call on inputs that are already on the GPU.

Keys of a case:
  op                 rotary, rotary_append, key_weights, evict_plan, kv_compact
  dtype              "bf16" or "f32": storage of q, k, v
  batch, hq, hkv, d  requests, query heads, KV heads, head dim
  s_lo, s_hi         cached keys of a request, spread evenly in the logarithm and dealt
                     to the requests by the seed
  n_lo, n_hi         new tokens of a request, spread in the same way (0: n = S, a prompt)
  axes, cyclic       position axes; a frequency's axis by contiguous sections or in turn
  rot, interleaved   rotated dims, and whether a pair's dims are neighbours
  fused              q, k and v are slices of one projection's rows
  sinks, partial     sink logits; only a part of the rows counts (accepted drafts)
  keep, first, recent  keys to keep at most, of which the first and the latest always
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 16
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
DEV = "cuda"


# ------------------------------------------------------------------ the cases

def _rotary(name, rows, hq, hkv, d, **kw):
    return dict(name=name, op="rotary", rows=rows, hq=hq, hkv=hkv, d=d,
                **{**dict(dtype="bf16", axes=1, cyclic=False, rot=d, interleaved=False, fused=False), **kw})


def _cache(name, op, batch, hq, hkv, d, s_lo, s_hi, **kw):
    c = dict(name=name, op=op, batch=batch, hkv=hkv, d=d, s_lo=s_lo, s_hi=s_hi, dtype="bf16")
    if op == "rotary_append":
        c.update(hq=hq, n_lo=1, n_hi=1, axes=1, cyclic=False, rot=d, interleaved=False, fused=False)
    if op == "key_weights":
        c.update(hq=hq, n_lo=1, n_hi=1, sinks=False, partial=False)
    if op in ("evict_plan", "kv_compact"):
        c.update(keep=1024, first=4, recent=64)
    c.update(kw)
    return c


def listed():
    return [
        # one token of one user: a launch's latency
        _rotary("rotary_one_token", 1, 32, 8, 128),
        # a prompt with images in it: three axes, q and k in the projection's own rows
        _rotary("rotary_image_prompt", 5461, 32, 8, 128, axes=3, fused=True),
        # the verify step of bench.py's batch: nine new tokens of each of 32 requests
        _cache("append_verify", "rotary_append", 32, 32, 8, 128, 2048, 16384, n_lo=9, n_hi=9),
        # prompts of a head-dim-64 model, ragged, three axes in turn over neighbouring pairs
        _cache("append_prompts", "rotary_append", 6, 64, 8, 64, 700, 4099, n_lo=0, n_hi=0, axes=3, cyclic=True,
               interleaved=True, fused=True),
        # one user's decode step: latency
        _cache("weights_one_token", "key_weights", 1, 32, 8, 128, 1501, 1501),
        # the verify step of bench.py's batch, the accepted rows counted
        _cache("weights_verify", "key_weights", 32, 32, 8, 128, 2048, 16384, n_lo=9, n_hi=9, partial=True),
        # whole prompts, every row's weights
        _cache("weights_prompt", "key_weights", 2, 32, 8, 128, 1300, 2531, n_lo=0, n_hi=0),
        # fp32 storage, head dim 64, sinks, a few ragged drafts
        _cache("weights_f32_sinks", "key_weights", 6, 64, 8, 64, 500, 4100, n_lo=1, n_hi=5, dtype="f32", sinks=True),
        # a batch's caches brought down to 4096 keys, once after the prompt
        _cache("plan_batch", "evict_plan", 32, 0, 8, 128, 2048, 16384, keep=4096, recent=512),
        # one very long session
        _cache("plan_long", "evict_plan", 1, 0, 8, 128, 131072, 131072, keep=16384, recent=2048),
        # the moves of the first of these
        _cache("compact_prompt", "kv_compact", 16, 0, 8, 128, 8192, 16384, keep=4096, recent=512),
        # every step's moves: nine new keys each, so nine leave
        _cache("compact_step", "kv_compact", 32, 0, 8, 128, 4105, 4105, keep=4096, recent=512),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "rotary_append", "key_weights", "key_weights", "evict_plan", "kv_compact"])
    d = rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    axes = rng.choice([1, 1, 2, 3, 4])
    turn = dict(axes=axes, cyclic=rng.random() < 0.5, rot=rng.choice([d, d, d // 2, d // 2 + 6]),
                interleaved=rng.random() < 0.4, fused=rng.random() < 0.5)
    if op == "rotary":
        c = _rotary("", _log(rng, 1, 6000), hq, hkv, d, dtype=dtype, **turn)
    elif op == "rotary_append":
        if rng.random() < 0.5:
            s = _log(rng, 20, 3000)
            c = _cache("", op, rng.randint(1, 6), hq, hkv, d, max(1, s // rng.randint(1, 6)), s, n_lo=0, n_hi=0,
                       dtype=dtype, **turn)
        else:
            s = _log(rng, 40, 8000)
            c = _cache("", op, _log(rng, 1, 48), hq, hkv, d, max(20, s // rng.randint(1, 8)), s, n_lo=1,
                       n_hi=rng.randint(1, 17), dtype=dtype, **turn)
    elif op == "key_weights":
        extra = dict(dtype=dtype, sinks=rng.random() < 0.4, partial=rng.random() < 0.5)
        if rng.random() < 0.3:
            s = _log(rng, 10, 1800)
            c = _cache("", op, rng.randint(1, 3), hq, hkv, d, max(1, s // rng.randint(1, 6)), s, n_lo=0, n_hi=0, **extra)
        else:
            s = _log(rng, 40, 12000)
            c = _cache("", op, _log(rng, 1, 32 if dtype == "bf16" else 12), hq, hkv, d, max(20, s // rng.randint(1, 8)), s,
                       n_lo=1, n_hi=rng.randint(1, 17), **extra)
    else:
        s = _log(rng, 40, 14000)
        keep = max(1, int(s * rng.uniform(0.05, 1.1)))
        c = _cache("", op, _log(rng, 1, 10 if dtype == "bf16" else 5), hq, hkv, d, max(1, s // rng.randint(1, 4)), s,
                   dtype=dtype, keep=keep, first=rng.randint(0, keep // 8), recent=rng.randint(0, keep // 2))
    del c["name"]
    return c


def _spread(lo, hi, count):
    """`count` whole numbers from lo to hi, even in their logarithm (the largest first)."""
    if count == 1:
        return [hi]
    return [int(round(hi * (lo / hi) ** (i / (count - 1)))) for i in range(count)]


def _lengths(case):
    """(S_i, n_i) of the case's requests, in an order that the seed then deals out."""
    S = _spread(case["s_lo"], case["s_hi"], case["batch"])
    if "n_lo" not in case:
        return S, [0] * len(S)
    if case["n_hi"] == 0:
        return S, list(S)
    n = _spread(case["n_lo"], case["n_hi"], case["batch"])
    return S, [min(a, b) for a, b in zip(n, S)]


def work(case):
    d, hkv, e = case["d"], case["hkv"], BYTES[case["dtype"]]
    if case["op"] == "rotary":
        x = case["rows"] * (case["hq"] + hkv)
        return {"bytes": 2 * x * d * e + 4 * case["axes"] * case["rows"], "flops": 3 * x * case["rot"]}
    S, n = _lengths(case)
    T, keys = sum(n), sum(S)
    if case["op"] == "rotary_append":
        x = T * (case["hq"] + hkv)
        return {"bytes": 2 * (x + T * hkv) * d * e + 4 * case["axes"] * T, "flops": 3 * x * case["rot"]}
    if case["op"] == "key_weights":
        # a prompt's rows see half of the keys on the average
        seen = sum(a * (b - a) + a * (a + 1) / 2 for b, a in zip(S, n))
        return {"bytes": keys * hkv * (d * e + 8) + T * case["hq"] * d * e + 8 * T * hkv,
                "flops": 2 * seen * case["hq"] * d}
    kept = sum(min(s, case["keep"]) for s in S)
    if case["op"] == "evict_plan":
        return {"bytes": hkv * (8 * keys + 4 * kept), "flops": hkv * keys}
    # the keys that leave the first slots, about in proportion
    moved = sum(min(s, case["keep"]) * max(0, s - case["keep"]) / s for s in S)
    return {"bytes": hkv * (4 * kept + 2 * moved * (2 * d * e + 8)), "flops": 0}


# ------------------------------------------------------------------ the inputs

def _axis_of(case):
    """The position axis of each frequency."""
    f, a = case["rot"] // 2, case["axes"]
    return [i % a if case["cyclic"] else i * a // f for i in range(f)]


def _positions(case, n, S, gen):
    """[axes][rows]: a request's text counts up on every axis; in its images the first
    axis stands still and the others run over the rows and columns of the patches."""
    n = torch.tensor(n, device=DEV)
    start = n.cumsum(0) - n
    req = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n)
    j = torch.arange(req.numel(), device=DEV) - start[req]
    at = torch.tensor(S, device=DEV)[req] - n[req] + j
    at = at + torch.randint(0, 100000, (n.numel(),), generator=gen, device=DEV)[req]
    image = (at // 700) % 2 == 1
    width = 20 + torch.randint(0, 9, (1,), generator=gen, device=DEV)
    base, in_image = at // 700 * 700, at % 700
    each = [base, base + in_image // width, base + in_image % width, base + in_image // 50]
    return torch.stack([torch.where(image, x, at) for x in each[:case["axes"]]]).to(torch.int32)


def _paged(case, S, gen):
    blocks = [(s + BLOCK - 1) // BLOCK for s in S]
    total = sum(blocks) + 3
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(S), max(blocks)), -1, dtype=torch.int32, device=DEV)
    off = 0
    for i, b in enumerate(blocks):
        table[i, :b] = ids[off:off + b]
        off += b
    return table, total


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _rows_of(case, rows, heads, gen):
    """q, k (and v) rows of `heads` heads each, alone or as slices of one row."""
    t, d = DTYPE[case["dtype"]], case["d"]
    if not case.get("fused"):
        return [_randn((rows, h, d), t, gen) for h in heads]
    x = _randn((rows, sum(heads), d), t, gen)
    return list(x.split(heads, dim=1))


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    t, d, hkv, op = DTYPE[case["dtype"]], case["d"], case["hkv"], case["op"]
    s = dict(case)
    if op in ("rotary", "rotary_append"):
        f = case["rot"] // 2
        s["inv_freq"] = 10000.0 ** (-torch.arange(f, dtype=torch.float64, device=DEV) / f)
        s["axis"] = _axis_of(case)
        s["axis_index"] = torch.tensor(s["axis"], device=DEV)
    if op == "rotary":
        rows = case["rows"]
        # a prompt, or one row of each request where there are few
        s["positions"] = _positions(case, [rows], [rows + 5], gen)
        s["q"], s["k"], _ = _rows_of(case, rows, [case["hq"], hkv, hkv], gen)
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=t, device=DEV) for x in (s["q"], s["k"]))
        return s
    S, n = _lengths(case)
    deal = random.Random(seed)
    both = list(zip(S, n))
    deal.shuffle(both)
    S, n = [list(x) for x in zip(*both)]
    B, T = len(S), sum(n)
    s.update(S=S, n=n, total_keys=sum(S), total_q=T, max_seq_len=max(S), max_q_len=max(n))
    s["seq_lens"] = _int(S)
    s["q_start"] = _int([sum(n[:i]) for i in range(B + 1)])
    s["block_tables"], nb = _paged(case, S, gen)
    if op != "evict_plan":
        x = 16 // BYTES[case["dtype"]]
        s["k_cache"] = _randn((nb, hkv, d // x, BLOCK, x), t, gen)
    if op in ("rotary_append", "kv_compact"):
        s["v_cache"] = _randn((nb, hkv, d, BLOCK), t, gen)
    if op == "rotary_append":
        s["positions"] = _positions(case, n, S, gen)
        s["q"], s["k_new"], s["v_new"] = _rows_of(case, T, [case["hq"], hkv, hkv], gen)
        s["q_out"] = torch.empty(s["q"].shape, dtype=t, device=DEV)
        return s
    # the caches have lost keys before: half as many as they hold; ordinals rise over
    # the slots but for the ones that took freed slots
    seen = [a + a // 2 for a in S]
    s["num_tokens"] = _int(seen)
    s["key_weights"] = torch.exp(2.0 * torch.randn((nb, hkv, BLOCK), generator=gen, device=DEV) - 7.0)
    # a tenth of the keys was never looked at
    s["key_weights"] *= torch.rand((nb, hkv, BLOCK), generator=gen, device=DEV) > 0.1
    s["key_order"] = torch.zeros((nb, hkv, BLOCK), dtype=torch.int32, device=DEV)
    req, slot, cell = _cells(s)
    turn = torch.randint(0, min(S), (hkv,), generator=gen, device=DEV)
    Sr = s["seq_lens"].long()[req][:, None]
    rank = (slot[:, None] + turn) % Sr
    s["key_order"].view(-1)[cell] = (rank * s["num_tokens"].long()[req][:, None] // Sr).to(torch.int32)
    if op == "key_weights":
        # a head's queries lean to a direction that a few of the keys hold too
        lean = torch.randn((hkv, 1, d), generator=gen, device=DEV)
        q = torch.randn((T, hkv, case["hq"] // hkv, d), generator=gen, device=DEV) + 0.5 * lean
        s["q"] = q.reshape(T, case["hq"], d).to(t)
        held = torch.rand((nb, hkv, 1, BLOCK, 1), generator=gen, device=DEV) < 0.02
        lean = lean.view(1, hkv, d // x, 1, x).to(t)
        s["k_cache"] += held.to(t) * lean
        s["sink_logits"] = torch.randn((case["hq"],), generator=gen, device=DEV) if case["sinks"] else None
        rows = [deal.randint(1, a) for a in n] if case["partial"] else n
        s["num_rows"] = _int(rows) if case["partial"] else None
        return s
    if op == "kv_compact":
        s["source"], s["new_lens"] = _plain_plan(s)
        s["total_kept"] = sum(min(a, case["keep"]) for a in S)
    else:
        s["source"] = torch.empty((B, hkv, case["keep"]), dtype=torch.int32, device=DEV)
        s["new_lens"] = torch.empty((B,), dtype=torch.int32, device=DEV)
    return s


# ------------------------------------------------------------------ the plain forms

def _packed(lens, total):
    """The request and the place within it of each of `total` packed items."""
    lens = lens.long()
    req = torch.repeat_interleave(torch.arange(lens.numel(), device=lens.device), lens, output_size=total)
    return req, torch.arange(total, device=lens.device) - (lens.cumsum(0) - lens)[req]


def _cells(s):
    """Every cached key: its request, its slot, and its place in [num_blocks][Hkv][16]."""
    req, slot = _packed(s["seq_lens"], s["total_keys"])
    block = s["block_tables"].long()[req, slot // BLOCK]
    g = torch.arange(s["hkv"], device=slot.device)
    return req, slot, (block[:, None] * s["hkv"] + g) * BLOCK + (slot % BLOCK)[:, None]


def _plain_turn(s, x, cos, sin):
    """x [T][H][D] with its first `rot` dims turned by the rows' angles."""
    r, y = s["rot"], x.float()
    if s["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, y[..., r:]], dim=-1).to(x.dtype)


def _plain_angles(s):
    # far positions times a frequency lose their fraction of a turn in 32 bits
    angle = s["positions"].double().index_select(0, s["axis_index"]).t() * s["inv_freq"]
    return angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]


def _plain_append(s):
    cos, sin = _plain_angles(s)
    q, k = _plain_turn(s, s["q"], cos, sin), _plain_turn(s, s["k_new"], cos, sin)
    n = s["q_start"][1:] - s["q_start"][:-1]
    req, j = _packed(n, s["total_q"])
    p = (s["seq_lens"] - n).long()[req] + j
    block = s["block_tables"].long()[req, p // BLOCK]
    kc, vc = s["k_cache"], s["v_cache"]
    kc[block, :, :, p % BLOCK, :] = k.reshape(k.shape[0], kc.shape[1], kc.shape[2], kc.shape[4])
    vc[block, :, :, p % BLOCK] = s["v_new"]
    return q, kc, vc


def _plain_weights(s):
    kc, hkv = s["k_cache"], s["hkv"]
    group = s["hq"] // hkv
    table = s["block_tables"].long().clamp(min=0)
    k = kc[table].permute(0, 2, 1, 4, 3, 5).reshape(len(s["S"]), hkv, table.shape[1] * BLOCK, s["d"]).float()
    S, q0 = s["seq_lens"].long(), s["q_start"].long()
    n = q0[1:] - q0[:-1]
    j = torch.arange(s["max_q_len"], device=kc.device)
    counted = n if s["num_rows"] is None else torch.minimum(n, s["num_rows"].long())
    rows = (q0[:-1, None] + j).clamp(max=s["total_q"] - 1)
    q = s["q"][rows].float().reshape(len(s["S"]), -1, hkv, group, s["d"]).permute(0, 2, 1, 3, 4)
    score = torch.matmul(q.reshape(len(s["S"]), hkv, -1, s["d"]), k.transpose(2, 3)) / math.sqrt(s["d"])
    score = score.view(len(s["S"]), hkv, s["max_q_len"], group, -1)
    t = torch.arange(score.shape[-1], device=kc.device)
    last = (S - n)[:, None] + j  # a row's own position
    seen = (t <= last[..., None]) & (j < counted[:, None])[..., None] & (t < S[:, None, None])
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    sink = None if s["sink_logits"] is None else s["sink_logits"].view(1, hkv, 1, group, 1)
    if sink is not None:
        top = torch.maximum(top, sink)
    top = torch.where(top == -math.inf, 0.0, top)
    e = score.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    if sink is not None:
        total = total + (sink - top).exp()
    w = (e / torch.where(total == 0, 1.0, total)).sum((2, 3))
    req, slot, cell = _cells(s)
    w = w[req, :, slot]
    j = (slot - (S - n)[req])[:, None]
    weights, order = s["key_weights"].view(-1), s["key_order"].view(-1)
    weights[cell] = torch.where(j >= 0, w, weights[cell] + w)
    order[cell] = torch.where(j >= 0, (s["num_tokens"].long() - n)[req][:, None] + j, order[cell].long()).to(torch.int32)
    return s["key_weights"], s["key_order"]


def _plain_plan(s):
    keep, table = s["keep"], s["block_tables"].long().clamp(min=0)
    wide = max(table.shape[1] * BLOCK, keep)
    slot = torch.arange(wide, device=table.device)
    at = slot.clamp(max=table.shape[1] * BLOCK - 1)
    w, order = (x[table].permute(0, 2, 1, 3).flatten(2)[..., at] for x in (s["key_weights"], s["key_order"]))
    S = s["seq_lens"].long()[:, None, None]
    c = S.clamp(max=keep)
    always = (order < s["first"]) | (order >= s["num_tokens"].long()[:, None, None] - s["recent"])
    w = torch.where(slot >= S, -math.inf, torch.where(always, math.inf, w))
    ranked = torch.sort(w, dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(w, dtype=torch.bool).scatter_(2, ranked, (slot < c).expand_as(w))
    hole, mover = ~kept & (slot < c), kept & (slot >= c)
    movers = torch.zeros(w.shape[:2] + (wide + 1,), dtype=torch.int64, device=w.device)
    movers.scatter_(2, torch.where(mover, mover.cumsum(2) - 1, wide), slot.expand_as(w))
    source = torch.where(hole, movers.gather(2, (hole.cumsum(2) - 1).clamp(min=0)), slot)
    source = torch.where(slot < c, source, -1)[..., :keep]
    return source.to(torch.int32).contiguous(), c.view(-1).to(torch.int32)


def _plain_moves(s):
    req, to = _packed(s["new_lens"], s["total_kept"])
    source = s["source"].long()[req, :, to]
    n, g = (source != to[:, None]).nonzero(as_tuple=True)  # the keys that move
    req, to, source, table = req[n], to[n], source[n, g], s["block_tables"].long()
    block, at = table[req, source // BLOCK], source % BLOCK
    out, slot = table[req, to // BLOCK], to % BLOCK
    kc, vc, w, o = s["k_cache"], s["v_cache"], s["key_weights"], s["key_order"]
    # all is read before anything is written
    k, v, weight, order = kc[block, g, :, at], vc[block, g, :, at], w[block, g, at], o[block, g, at]
    kc[out, g, :, slot], vc[out, g, :, slot], w[out, g, slot], o[out, g, slot] = k, v, weight, order
    return kc, vc, w, o


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "rotary":
        cos, sin = _plain_angles(s)
        return _plain_turn(s, s["q"], cos, sin), _plain_turn(s, s["k"], cos, sin)
    return {"rotary_append": _plain_append, "key_weights": _plain_weights, "evict_plan": _plain_plan,
            "kv_compact": _plain_moves}[s["op"]](s)


def _run_own(s):
    import paper_2608_24004_amd as av

    if s["op"] == "rotary":
        return av.verify_rotary(s["q"], s["k"], s["positions"], s["inv_freq"], axes=s["axis"],
                                interleaved=s["interleaved"], q_out=s["q_out"], k_out=s["k_out"])
    if s["op"] == "rotary_append":
        q = av.verify_rotary_append(s["q"], s["k_new"], s["v_new"], s["positions"], s["inv_freq"], s["k_cache"],
                                    s["v_cache"], s["block_tables"], s["seq_lens"], s["q_start"], axes=s["axis"],
                                    interleaved=s["interleaved"], q_out=s["q_out"])
        return q, s["k_cache"], s["v_cache"]
    if s["op"] == "key_weights":
        bounds = dict(max_q_len=s["max_q_len"], max_seq_len=s["max_seq_len"])
        if "workspace" not in s:  # a program keeps one
            size = av.key_weights_workspace_size(s["q"], s["k_cache"], s["block_tables"], **bounds)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
        av.verify_key_weights(s["q"], s["k_cache"], s["key_weights"], s["key_order"], s["block_tables"], s["seq_lens"],
                              s["q_start"], num_rows=s["num_rows"], num_tokens=s["num_tokens"],
                              sinks=s["sink_logits"], workspace=s["workspace"], **bounds)
        return s["key_weights"], s["key_order"]
    if s["op"] == "evict_plan":
        return av.verify_evict_plan(s["key_weights"], s["key_order"], s["block_tables"], s["seq_lens"],
                                    max_keys=s["keep"], keep_first=s["first"], keep_recent=s["recent"],
                                    max_seq_len=s["max_seq_len"], num_tokens=s["num_tokens"], source=s["source"],
                                    new_lens=s["new_lens"])
    av.verify_kv_compact(s["k_cache"], s["v_cache"], s["block_tables"], s["source"], s["new_lens"],
                         key_weights=s["key_weights"], key_order=s["key_order"])
    return s["k_cache"], s["v_cache"], s["key_weights"], s["key_order"]


# ------------------------------------------------------------------ 64 bits

def _exact_turn(s, x):
    """Each pair as a complex number times e^(i angle)."""
    f = s["rot"] // 2
    y = x.double().clone()
    for i in range(f):
        a, b = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + f)
        angle = s["positions"][s["axis"][i]].double() * float(s["inv_freq"][i])
        z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        y[..., a], y[..., b] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "rotary":
        return _exact_turn(s, s["q"]), _exact_turn(s, s["k"])
    if op == "evict_plan":
        return None
    table = s["block_tables"].cpu().tolist()
    S = s["S"]
    blocks = [torch.tensor(table[i][:(S[i] + BLOCK - 1) // BLOCK], device=DEV) for i in range(len(S))]
    hkv, d = s["hkv"], s["d"]
    kc = s["k_cache"]
    if op == "rotary_append":
        q, k = _exact_turn(s, s["q"]), _exact_turn(s, s["k_new"])
        kc, vc = kc.double(), s["v_cache"].double()
        start = 0
        for i, n in enumerate(s["n"]):
            for j in range(n):
                p, r = S[i] - n + j, start + j
                b = table[i][p // BLOCK]
                kc[b, :, :, p % BLOCK] = k[r].view(hkv, kc.shape[2], kc.shape[4])
                vc[b, :, :, p % BLOCK] = s["v_new"][r].double()
            start += n
        return q, kc, vc
    if op == "key_weights":
        out = s["key_weights"].double()
        start = 0
        group = s["hq"] // hkv
        for i, n in enumerate(s["n"]):
            count = n if s["num_rows"] is None else int(s["num_rows"][i])
            pos = torch.arange(S[i] - n, S[i] - n + count, device=DEV).repeat_interleave(group)
            hidden = torch.arange(S[i], device=DEV) > pos[:, None]
            for g in range(hkv):
                # [blocks][D/x][16][x] -> [keys][D]
                k = kc[blocks[i], g].transpose(1, 2).reshape(-1, d)[:S[i]].double()
                q = s["q"][start:start + count, g * group:(g + 1) * group].reshape(-1, d).double()
                x = (q @ k.t() / math.sqrt(d)).masked_fill(hidden, -math.inf)
                if s["sink_logits"] is not None:
                    last = s["sink_logits"][g * group:(g + 1) * group].double().repeat(count)[:, None]
                    x = torch.cat([x, last], dim=1)
                w = torch.softmax(x, dim=1)[:, :S[i]].sum(0)
                line = out[blocks[i], g].reshape(-1)
                line[S[i] - n:S[i]] = 0
                line[:S[i]] += w
                out[blocks[i], g] = line.view(-1, BLOCK)
            start += n
        return out, None
    # kv_compact: a request's keys in a line, the sources picked from it
    outs = [kc.double(), s["v_cache"].double(), s["key_weights"].double()]
    for i in range(len(S)):
        c = min(S[i], case["keep"])
        b = blocks[i]
        for g in range(hkv):
            src = s["source"][i, g, :c].long()
            for x, dim in ((outs[0], 2), (outs[1], 2), (outs[2], 1)):
                # the slot axis first, then the blocks and slots as one line
                tile = x[b, g].movedim(dim, 1)
                line = tile.reshape((-1,) + tile.shape[2:])
                line = torch.cat([line[src], line[c:]])
                x[b, g] = line.view(tile.shape).movedim(1, dim)
    return outs[0], outs[1], outs[2], None
