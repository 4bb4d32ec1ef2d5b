"""The calls around the verify step of a batch of agents, as measured cases.

Agents of one kind begin with the same instructions and tool descriptions, answer in a
grammar and are kept from repeating themselves.  A serving engine that decodes a batch
of them norms and rotates the new tokens' queries and keys (and appends the keys and
values), attends to the prefix that requests share once for all of them, and changes
the logits by penalties, biases and grammar masks before it accepts drafts from them;
the penalties read counts of the tokens that stand, which are kept on the GPU.  A case
is one such call on inputs that are already on the GPU.

Keys of a case:
  op                 norm_rotary, norm_rotary_append, shared_attention, adjust_logits, count_tokens
  dtype              "bf16" or "f32": storage of q, k, v or of the logits
  batch, hq, hkv, d  requests, query heads, KV heads, head dim
  rows               packed rows of a norm_rotary case
  n_lo, n_hi         new tokens of a request, spread evenly in the logarithm and dealt to
                     the requests by the seed (n_hi 0: as many as cached keys, a prompt)
  s_lo, s_hi         a request's cached keys, behind its group's prefix if there is one
  groups, p_lo, p_hi groups of requests, and the keys of their common prefixes
  axes, cyclic       position axes; a frequency's axis by contiguous sections or in turn
  rot, interleaved   rotated dims, and whether a pair's dims are neighbours
  fused              q, k and v are slices of one projection's rows
  sinks              sink logits
  vocab, history     vocabulary entries, tokens that a request has had
  penalties, biases, masks   of the logits: truth value, biased tokens, truth value
  prompt             counted tokens belong to prompts
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
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def _norm(name, rows, hq, hkv, d, **kw):
    return dict(name=name, op="norm_rotary", rows=rows, hq=hq, hkv=hkv, d=d,
                **{**dict(dtype="bf16", axes=1, cyclic=False, rot=d, interleaved=False, fused=False), **kw})


def _append(name, batch, hq, hkv, d, s_lo, s_hi, **kw):
    return dict(name=name, op="norm_rotary_append", batch=batch, hq=hq, hkv=hkv, d=d, s_lo=s_lo, s_hi=s_hi,
                **{**dict(dtype="bf16", n_lo=1, n_hi=1, axes=1, cyclic=False, rot=d, interleaved=False, fused=False), **kw})


def _shared(name, batch, hq, hkv, d, s_lo, s_hi, p_lo, p_hi, **kw):
    return dict(name=name, op="shared_attention", batch=batch, hq=hq, hkv=hkv, d=d, s_lo=s_lo, s_hi=s_hi, p_lo=p_lo,
                p_hi=p_hi, **{**dict(dtype="bf16", groups=1, n_lo=1, n_hi=1, sinks=False), **kw})


def _adjust(name, batch, vocab, **kw):
    return dict(name=name, op="adjust_logits", batch=batch, vocab=vocab,
                **{**dict(dtype="bf16", n_lo=1, n_hi=1, history=2000, penalties=True, biases=0, masks=False), **kw})


def _count(name, batch, vocab, n_lo, n_hi, **kw):
    return dict(name=name, op="count_tokens", batch=batch, vocab=vocab, n_lo=n_lo, n_hi=n_hi,
                **{**dict(dtype="bf16", history=2000, prompt=False), **kw})


def listed():
    return [
        # one token of one user: a launch's latency
        _norm("norm_one_token", 1, 32, 8, 128),
        # a prompt's rows, q and k in the projection's own rows
        _norm("norm_prompt", 5461, 32, 8, 128, fused=True),
        # the verify step of bench.py's batch: nine new tokens of each of 32 requests
        _append("norm_append_verify", 32, 32, 8, 128, 2048, 16384, n_lo=9, n_hi=9, fused=True),
        # ragged prompts, half of the dims rotated, neighbouring pairs, three axes in turn
        _append("norm_append_prompts", 6, 64, 8, 64, 700, 4099, n_lo=0, n_hi=0, axes=3, cyclic=True, rot=32,
                interleaved=True),
        # two requests behind a short common start, in fp32: latency
        _shared("shared_two_f32", 2, 32, 8, 128, 33, 60, 333, 333, dtype="f32"),
        # one token of each of 64 agents with the same instructions
        _shared("shared_decode", 64, 32, 8, 128, 130, 1500, 8192, 8192),
        # the verify step of 32 of them, nine rows each, later in their work
        _shared("shared_verify", 32, 32, 8, 128, 512, 4096, 8192, 8192, n_lo=9, n_hi=9),
        # three kinds of agents, ragged drafts, head dim 64 with sinks
        _shared("shared_kinds", 24, 64, 8, 64, 75, 2077, 1205, 6002, groups=3, n_lo=1, n_hi=17, sinks=True),
        # the verify step's logits, all that a request may ask for
        _adjust("adjust_verify", 32, 151936, n_lo=9, n_hi=9, biases=40, masks=True),
        # single tokens, an odd vocabulary in fp32, penalties alone
        _adjust("adjust_odd_f32", 5, 50003, dtype="f32"),
        # the tokens that a verify step emits
        _count("count_step", 32, 151936, 1, 9),
        # the prompts of newly arrived requests
        _count("count_prompts", 8, 151936, 2048, 16384, history=0, prompt=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm_rotary", "norm_rotary_append", "shared_attention", "shared_attention", "adjust_logits",
                     "adjust_logits", "count_tokens"])
    d = rng.choice([64, 128])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 8])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    turn = dict(axes=rng.choice([1, 1, 2, 3, 4]), cyclic=rng.random() < 0.5, rot=rng.choice([d, d, d // 2, d // 2 + 6]),
                interleaved=rng.random() < 0.4, fused=rng.random() < 0.5)
    if op == "norm_rotary":
        c = _norm("", _log(rng, 1, 6000), hq, hkv, d, dtype=dtype, **turn)
    elif op == "norm_rotary_append":
        if rng.random() < 0.5:
            s = _log(rng, 20, 3000)
            c = _append("", rng.randint(1, 6), hq, hkv, d, max(1, s // rng.randint(1, 6)), s, n_lo=0, n_hi=0,
                        dtype=dtype, **turn)
        else:
            s = _log(rng, 40, 8000)
            c = _append("", _log(rng, 1, 48), hq, hkv, d, max(20, s // rng.randint(1, 8)), s, n_lo=1,
                        n_hi=rng.randint(1, 17), dtype=dtype, **turn)
    elif op == "shared_attention":
        batch = _log(rng, 2, 64)
        s, p = _log(rng, 20, 3000), _log(rng, 16, 8192)
        n = rng.randint(1, 17)
        while batch * n > 288:
            n = max(1, n // 2)
        kinds = rng.randint(1, min(4, batch // 2))
        c = _shared("", batch, hq, hkv, d, max(18, s // rng.randint(1, 8)), max(18, s),
                    max(1, p // rng.randint(1, 4)) if kinds > 1 else p, p, groups=kinds, n_lo=1, n_hi=n, dtype=dtype,
                    sinks=rng.random() < 0.4)
        if dtype == "f32":  # 16 times the work of a product
            c["p_lo"], c["p_hi"] = (c["p_lo"] + 3) // 4, (c["p_hi"] + 3) // 4
    elif op == "adjust_logits":
        n = rng.randint(1, 17)
        batch = max(1, min(_log(rng, 1, 64), 288 // n))
        c = _adjust("", batch, _log(rng, 300, 150000), dtype=dtype, n_lo=1, n_hi=n, history=_log(rng, 1, 8000),
                    penalties=rng.random() < 0.8, biases=rng.choice([0, 3, 40, 300]), masks=rng.random() < 0.6)
        if dtype == "f32":
            c["batch"] = (c["batch"] + 1) // 2
    elif rng.random() < 0.5:
        c = _count("", _log(rng, 1, 64), _log(rng, 300, 150000), 1, rng.randint(1, 17), history=_log(rng, 1, 8000))
    else:
        n = _log(rng, 20, 16000)
        c = _count("", rng.randint(1, 8), _log(rng, 300, 150000), max(1, n // rng.randint(1, 8)), n, history=0, prompt=True)
    del c["name"]
    return c


def _spread(lo, hi, count):
    """`count` whole numbers from lo to hi, even in their logarithm (the largest first)."""
    if count == 1:
        return [hi]
    return [int(round(hi * (lo / hi) ** (i / (count - 1)))) for i in range(count)]


def _new(case):
    """The new tokens of the case's requests."""
    return _spread(case["n_lo"], case["n_hi"], case["batch"])


def _lengths(case):
    """(cached keys behind the prefix, new tokens) of the case's requests, in an order
    that the seed then deals out."""
    S = _spread(case["s_lo"], case["s_hi"], case["batch"])
    if case["n_hi"] == 0:
        return S, list(S)
    return S, [min(a, b) for a, b in zip(_new(case), S)]


def _groups(case):
    """The first request of each group (and the end), and the groups' prefixes."""
    k = case["groups"]
    return [case["batch"] * i // k for i in range(k + 1)], _spread(case["p_lo"], case["p_hi"], k)


def _words(vocab):
    return (vocab + 31) // 32


def work(case):
    op = case["op"]
    if op in ("adjust_logits", "count_tokens"):
        n, vocab, B = _new(case), case["vocab"], case["batch"]
        T = sum(n)
        if op == "count_tokens":  # the token, its count and its bit
            return {"bytes": T * (4 + 8 + 8), "flops": T}
        total = 2 * T * vocab * BYTES[case["dtype"]]
        if case["penalties"]:
            total += B * (8 * _words(vocab) + 4 * min(case["history"], vocab))
        total += 8 * B * case["biases"] + (4 * T * _words(vocab) if case["masks"] else 0)
        return {"bytes": total, "flops": 6 * B * min(case["history"], vocab) * case["penalties"] * T // B}
    d, hq, hkv, e = case["d"], case["hq"], case["hkv"], BYTES[case["dtype"]]
    if op == "norm_rotary":
        x = case["rows"] * (hq + hkv)
        return {"bytes": 2 * x * d * e + 4 * case["axes"] * case["rows"], "flops": x * (3 * case["rot"] + 4 * d)}
    S, n = _lengths(case)
    T = sum(n)
    if op == "norm_rotary_append":
        x = T * (hq + hkv)
        return {"bytes": 2 * (x + T * hkv) * d * e + 4 * case["axes"] * T, "flops": x * (3 * case["rot"] + 4 * d)}
    first, P = _groups(case)
    # a common block counts once; a prefix's last, partial block belongs to each request
    keys = sum(S) + sum(p // BLOCK * BLOCK + (first[k + 1] - first[k]) * (p % BLOCK) for k, p in enumerate(P))
    mean = sum(p * (first[k + 1] - first[k]) for k, p in enumerate(P)) / case["batch"]
    seen = sum(a * (mean + b - a) + a * (a + 1) / 2 for b, a in zip(S, n))
    return {"bytes": 2 * keys * hkv * d * e + 2 * T * hq * d * e, "flops": 4 * seen * hq * d}


# ------------------------------------------------------------------ the inputs

def _axis_of(case):
    """The position axis of each frequency."""
    f, a = case["rot"] // 2, case["axes"]
    return [i % a if case["cyclic"] else i * a // f for i in range(f)]


def _positions(case, n, S, gen):
    """[axes][rows]: text counts up on every axis; in an image the first axis stands
    still and the others run over the rows and columns of its patches."""
    n = torch.tensor(n, device=DEV)
    start = n.cumsum(0) - n
    req = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n)
    at = torch.tensor(S, device=DEV)[req] - n[req] + torch.arange(req.numel(), device=DEV) - start[req]
    at = at + torch.randint(0, 30000, (n.numel(),), generator=gen, device=DEV)[req]
    image = (at // 600) % 2 == 1
    width = 18 + torch.randint(0, 11, (1,), generator=gen, device=DEV)
    base, inside = at // 600 * 600, at % 600
    each = [base, base + inside // width, base + inside % width, base + inside // 40]
    return torch.stack([torch.where(image, x, at) for x in each[:case["axes"]]]).to(torch.int32)


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)


def _rows_of(case, rows, heads, gen):
    """q, k (and v) rows of `heads` heads each, alone or as slices of one row.  A head's
    rows differ in length, as a projection's do."""
    t, d = DTYPE[case["dtype"]], case["d"]
    x = torch.randn((rows, sum(heads), d), generator=gen, device=DEV)
    x = (x * torch.exp(0.7 * torch.randn((rows, sum(heads), 1), generator=gen, device=DEV))).to(t)
    parts = x.split(heads, dim=1)
    return list(parts) if case["fused"] else [p.contiguous() for p in parts]


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _starts(n):
    out = [0]
    for a in n:
        out.append(out[-1] + a)
    return out


def _tables(first, P, S, gen):
    """Block tables of requests of S keys whose group's whole prefix blocks are the same."""
    blocks = [(s + BLOCK - 1) // BLOCK for s in S]
    ids = iter(torch.randperm(sum(blocks) + 3, generator=gen, device=DEV).tolist())
    table = []
    for k, p in enumerate(P):
        common = [next(ids) for _ in range(p // BLOCK)]
        table += [common + [next(ids) for _ in range(blocks[i] - len(common))] for i in range(first[k], first[k + 1])]
    wide = max(blocks)
    used = max(max(row) for row in table) + 1
    return _int([row + [-1] * (wide - len(row)) for row in table]), used


def _history(case, gen):
    """[B][history] tokens, the common ones often, as text has them."""
    u = torch.rand((case["batch"], case["history"]), generator=gen, device=DEV, dtype=torch.float64)
    return ((case["vocab"] ** u - 1.0) / (case["vocab"] - 1.0) * case["vocab"]).long().clamp(max=case["vocab"] - 1)


def _pack(bits):
    """[..., V] truth values as int32 words of 32 tokens, the lowest bit first."""
    wide = _words(bits.shape[-1]) * 32
    x = torch.zeros(bits.shape[:-1] + (wide,), dtype=torch.int64, device=bits.device)
    x[..., :bits.shape[-1]] = bits
    x = (x.view(bits.shape[:-1] + (-1, 32)) << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(x >= 1 << 31, x - (1 << 32), x).to(torch.int32)


def _unpack(words, vocab):
    bits = (words.long()[..., None] >> torch.arange(32, device=words.device)) & 1
    return bits.flatten(-2)[..., :vocab] != 0


def _prepare_tokens(s, case, gen, deal):
    n, B, vocab = _new(case), case["batch"], case["vocab"]
    deal.shuffle(n)
    T = sum(n)
    s.update(n=n, total=T, slots=torch.randperm(B + 2, generator=gen, device=DEV)[:B].to(torch.int32))
    s["starts"] = _int(_starts(n))
    # half of a request's tokens came with its prompt
    past = _history(case, gen)
    half = case["history"] // 2
    slot = s["slots"].long()[:, None]
    counts = torch.zeros((B + 2, vocab), dtype=torch.int32, device=DEV)
    counts.index_put_((slot.expand_as(past[:, half:]), past[:, half:]), _int(1), accumulate=True)
    prompt = torch.zeros((B + 2, vocab), dtype=torch.bool, device=DEV)
    prompt[slot.expand_as(past[:, :half]), past[:, :half]] = True
    s["counts"], s["seen"] = counts, torch.stack([_pack(prompt), _pack(counts > 0)], dim=1).contiguous()
    fresh = dict(case, batch=1, history=T)
    s["tokens"] = _history(fresh, gen)[0].to(torch.int32)
    if case["op"] == "count_tokens":
        if not case["prompt"]:
            # a verify step's emitted tokens, -1 behind them
            rows = [deal.randint(1, a) for a in n]
            s["num"] = _int(rows)
            req, j = _packed(s["starts"][1:] - s["starts"][:-1], T)
            s["tokens"] = torch.where(j < s["num"].long()[req], s["tokens"], -1)
        else:
            s["num"] = None
        return s
    s["logits"] = _randn((T, vocab), DTYPE[case["dtype"]], gen) * 3
    s["out"] = torch.empty_like(s["logits"])
    for name, base, spread in (("repetition", 1.0, 0.3), ("frequency", 0.0, 0.5), ("presence", 0.0, 0.8)):
        s[name] = base + spread * torch.rand((B,), generator=gen, device=DEV) if case["penalties"] else None
    if case["biases"]:
        m = case["biases"]
        s["bias_start"] = _int([i * m for i in range(B + 1)])
        s["bias_tokens"] = torch.randint(0, vocab, (B * m,), generator=gen, device=DEV).to(torch.int32)
        s["bias_values"] = 4 * torch.randn((B * m,), generator=gen, device=DEV)
    if case["masks"]:
        # grammar states: inside a string nearly all tokens, elsewhere few; a row in
        # eight is free
        states = max(2, T // 2)
        share = torch.tensor([0.97, 0.002, 0.1], device=DEV)[torch.arange(states, device=DEV) % 3]
        allowed = torch.rand((states, vocab), generator=gen, device=DEV) < share[:, None]
        s["mask"] = _pack(allowed)
        at = torch.randint(0, states, (T,), generator=gen, device=DEV)
        s["mask_rows"] = torch.where(torch.rand((T,), generator=gen, device=DEV) < 0.125, -1, at).to(torch.int32)
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    deal = random.Random(seed)
    op = case["op"]
    s = dict(case)
    if op in ("adjust_logits", "count_tokens"):
        return _prepare_tokens(s, case, gen, deal)
    t, d, hkv = DTYPE[case["dtype"]], case["d"], case["hkv"]
    if op != "shared_attention":
        f = case["rot"] // 2
        s["inv_freq"] = 10000.0 ** (-torch.arange(f, dtype=torch.float64, device=DEV) / f)
        s["axis"] = _axis_of(case)
        s["axis_index"] = torch.tensor(s["axis"], device=DEV)
        s["q_weight"], s["k_weight"] = (1 + 0.2 * torch.randn((d,), generator=gen, device=DEV) for _ in range(2))
    if op == "norm_rotary":
        rows = case["rows"]
        s["positions"] = _positions(case, [rows], [rows + 5], gen)
        s["q"], s["k"], _ = _rows_of(case, rows, [case["hq"], hkv, hkv], gen)
        s["q_out"], s["k_out"] = (torch.empty(x.shape, dtype=t, device=DEV) for x in (s["q"], s["k"]))
        return s
    S, n = _lengths(case)
    both = list(zip(S, n))
    deal.shuffle(both)
    S, n = [list(x) for x in zip(*both)]
    B, T = len(S), sum(n)
    first, P = _groups(case) if op == "shared_attention" else (list(range(B + 1)), [0] * B)
    if op == "shared_attention":
        for k, p in enumerate(P):
            for i in range(first[k], first[k + 1]):
                S[i] += p
        s.update(first=first, P=P, max_prefix_len=max(P), group_start=_int(first), prefix_lens=_int(P))
    s.update(S=S, n=n, total_q=T, max_seq_len=max(S), max_q_len=max(n), seq_lens=_int(S), q_start=_int(_starts(n)))
    s["block_tables"], nb = _tables(first, P, S, gen)
    x = 16 // BYTES[case["dtype"]]
    s["k_cache"] = _randn((nb, hkv, d // x, BLOCK, x), t, gen)
    s["v_cache"] = _randn((nb, hkv, d, BLOCK), t, gen)
    if op == "norm_rotary_append":
        s["positions"] = _positions(case, n, S, gen)
        s["q"], s["k_new"], s["v_new"] = _rows_of(case, T, [case["hq"], hkv, hkv], gen)
        s["q_out"] = torch.empty(s["q"].shape, dtype=t, device=DEV)
        return s
    # a head's queries lean to a direction that a few of the keys hold too
    lean = torch.randn((hkv, 1, d), generator=gen, device=DEV)
    q = torch.randn((T, hkv, case["hq"] // hkv, d), generator=gen, device=DEV) + 0.5 * lean
    s["q"] = q.reshape(T, case["hq"], d).to(t)
    held = torch.rand((nb, hkv, 1, BLOCK, 1), generator=gen, device=DEV) < 0.02
    s["k_cache"] += held.to(t) * lean.view(1, hkv, d // x, 1, x).to(t)
    s["sink_logits"] = torch.randn((case["hq"],), generator=gen, device=DEV) if case["sinks"] else None
    s["out"] = torch.empty_like(s["q"])
    return s


# ------------------------------------------------------------------ the plain forms

def _packed(lens, total):
    """The request and the place within it of each of `total` packed items."""
    lens = lens.long()
    req = torch.repeat_interleave(torch.arange(lens.numel(), device=lens.device), lens, output_size=total)
    return req, torch.arange(total, device=lens.device) - (lens.cumsum(0) - lens)[req]


def _plain_norm_turn(s, x, weight, cos, sin):
    """x [T][H][D], each head at the length that its weights give it, its first `rot`
    dims turned by the rows' angles."""
    r, y = s["rot"], x.float()
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight
    if s["interleaved"]:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([turned, y[..., r:]], dim=-1).to(x.dtype)


def _plain_norm(s, keys):
    # far positions times a frequency lose their fraction of a turn in 32 bits
    angle = s["positions"].double().index_select(0, s["axis_index"]).t() * s["inv_freq"]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    return _plain_norm_turn(s, s["q"], s["q_weight"], cos, sin), _plain_norm_turn(s, s[keys], s["k_weight"], cos, sin)


def _plain_append(s):
    q, k = _plain_norm(s, "k_new")
    n = s["q_start"][1:] - s["q_start"][:-1]
    req, j = _packed(n, s["total_q"])
    p = (s["seq_lens"] - n).long()[req] + j
    block = s["block_tables"].long()[req, p // BLOCK]
    kc, vc = s["k_cache"], s["v_cache"]
    kc[block, :, :, p % BLOCK, :] = k.reshape(k.shape[0], kc.shape[1], kc.shape[2], kc.shape[4])
    vc[block, :, :, p % BLOCK] = s["v_new"]
    return q, kc, vc


def _plain_attention(s):
    hkv, d, B, group = s["hkv"], s["d"], len(s["S"]), s["hq"] // s["hkv"]
    table = s["block_tables"].long().clamp(min=0)
    k = s["k_cache"][table].permute(0, 2, 1, 4, 3, 5).reshape(B, hkv, table.shape[1] * BLOCK, d).float()
    v = s["v_cache"][table].permute(0, 2, 1, 4, 3).reshape(B, hkv, table.shape[1] * BLOCK, d).float()
    S, q0 = s["seq_lens"].long(), s["q_start"].long()
    n = q0[1:] - q0[:-1]
    j = torch.arange(s["max_q_len"], device=q0.device)
    rows = (q0[:-1, None] + j).clamp(max=s["total_q"] - 1)
    q = s["q"][rows].float().reshape(B, -1, hkv, group, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, d)
    score = torch.matmul(q, k.transpose(2, 3)).view(B, hkv, s["max_q_len"], group, -1) / math.sqrt(d)
    t = torch.arange(score.shape[-1], device=q0.device)
    last = (S - n)[:, None] + j  # a row's own position
    seen = (t <= last[..., None]) & (t < S[:, None, None])
    score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    sink = None if s["sink_logits"] is None else s["sink_logits"].view(1, hkv, 1, group, 1)
    if sink is not None:
        top = torch.maximum(top, sink)
    e = score.sub_(top).exp_()
    total = e.sum(-1, keepdim=True)
    if sink is not None:
        total = total + (sink - top).exp()
    o = torch.matmul(e.view(B, hkv, -1, e.shape[-1]), v).view(B, hkv, -1, group, d) / total
    o = o.permute(0, 2, 1, 3, 4).reshape(B, -1, s["hq"], d)
    req, at = _packed(n, s["total_q"])
    return o[req, at].to(s["q"].dtype)


def _plain_adjust(s):
    x, vocab = s["logits"].float(), s["vocab"]
    n = s["starts"][1:] - s["starts"][:-1]
    req, j = _packed(n, s["total"])
    if s["penalties"]:
        slot = s["slots"].long()
        count, prompt = s["counts"][slot], _unpack(s["seen"][slot, 0], vocab)
        # row j stands behind the drafts 1 .. j of its request
        at = torch.arange(max(s["n"]), device=x.device)
        behind = (at >= 1) & (at <= j[:, None])
        draft = s["tokens"].long()[(s["starts"].long()[req, None] + at).clamp(max=s["total"] - 1)]
        c = count[req].float()
        c.scatter_add_(1, draft, behind.float())
        r, f, p = (s[k][req, None] for k in ("repetition", "frequency", "presence"))
        x = torch.where(prompt[req] | (c > 0), torch.where(x > 0, x / r, x * r), x)
        x = x - f * c - torch.where(c > 0, p, 0.0)
    if s["biases"]:
        bias = torch.zeros((len(s["n"]), vocab), device=x.device)
        owner, _ = _packed(s["bias_start"][1:] - s["bias_start"][:-1], s["bias_tokens"].numel())
        bias.index_put_((owner, s["bias_tokens"].long()), s["bias_values"], accumulate=True)
        x = x + bias[req]
    if s["masks"]:
        row = s["mask_rows"].long()
        allowed = _unpack(s["mask"][row.clamp(min=0)], vocab) | (row < 0)[:, None]
        x = x.masked_fill_(~allowed, -math.inf)
    return x.to(s["logits"].dtype)


def _plain_count(s):
    vocab = s["vocab"]
    req, j = _packed(s["starts"][1:] - s["starts"][:-1], s["total"])
    tok = s["tokens"].long()
    counted = (tok >= 0) & (tok < vocab)
    if s["num"] is not None:
        counted &= j < s["num"].long()[req]
    slot = s["slots"].long()[req]
    hits = torch.zeros_like(s["counts"])
    hits.index_put_((slot, tok.clamp(0, vocab - 1)), counted.to(torch.int32), accumulate=True)
    s["seen"][:, 0 if s["prompt"] else 1] |= _pack(hits > 0)
    if not s["prompt"]:
        s["counts"] += hits
    return s["counts"], s["seen"]


# ------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "norm_rotary":
        return _plain_norm(s, "k")
    return {"norm_rotary_append": _plain_append, "shared_attention": _plain_attention, "adjust_logits": _plain_adjust,
            "count_tokens": _plain_count}[s["op"]](s)


def _run_own(s):
    import paper_2608_24004_amd as av

    op = s["op"]
    if op == "norm_rotary":
        return av.verify_norm_rotary(s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["q_weight"],
                                     k_weight=s["k_weight"], eps=EPS, axes=s["axis"], interleaved=s["interleaved"],
                                     q_out=s["q_out"], k_out=s["k_out"])
    if op == "norm_rotary_append":
        q = av.verify_norm_rotary_append(s["q"], s["k_new"], s["v_new"], s["positions"], s["inv_freq"], s["k_cache"],
                                         s["v_cache"], s["block_tables"], s["seq_lens"], s["q_start"],
                                         q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, axes=s["axis"],
                                         interleaved=s["interleaved"], q_out=s["q_out"])
        return q, s["k_cache"], s["v_cache"]
    if op == "shared_attention":
        bounds = dict(max_q_len=s["max_q_len"], max_seq_len=s["max_seq_len"], max_prefix_len=s["max_prefix_len"])
        if "workspace" not in s:  # a program keeps one
            size = av.attention_shared_workspace_size(s["q"], s["k_cache"], s["block_tables"], num_groups=s["groups"],
                                                      **bounds)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
        return av.verify_attention_shared(s["q"], s["k_cache"], s["v_cache"], s["block_tables"], s["seq_lens"],
                                          s["q_start"], s["group_start"], s["prefix_lens"], sinks=s["sink_logits"],
                                          out=s["out"], workspace=s["workspace"], **bounds)
    if op == "adjust_logits":
        return av.verify_adjust_logits(s["logits"], s["tokens"], s["starts"], counts=s["counts"], seen=s["seen"],
                                       slots=s["slots"], repetition=s["repetition"], frequency=s["frequency"],
                                       presence=s["presence"], bias_start=s.get("bias_start"),
                                       bias_tokens=s.get("bias_tokens"), bias_values=s.get("bias_values"),
                                       mask=s.get("mask"), mask_rows=s.get("mask_rows"), out=s["out"])
    av.verify_count_tokens(s["counts"], s["seen"], s["tokens"], s["starts"], num_tokens=s["num"], slots=s["slots"],
                           prompt=s["prompt"])
    return s["counts"], s["seen"]


# ------------------------------------------------------------------ 64 bits

def _exact_norm_turn(s, x, weight):
    """Each pair as a complex number times e^(i angle)."""
    f = s["rot"] // 2
    y = x.double()
    y = y / (y.square().sum(-1, keepdim=True) / s["d"] + EPS).sqrt() * weight.double()
    for i in range(f):
        a, b = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + f)
        angle = s["positions"][s["axis"][i]].double() * float(s["inv_freq"][i])
        z = torch.complex(y[..., a], y[..., b]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        y[..., a], y[..., b] = z.real, z.imag
    return y


def _exact_adjust(s):
    out = s["logits"].double()
    slots, tokens, starts, vocab = s["slots"].tolist(), s["tokens"].tolist(), s["starts"].tolist(), s["vocab"]
    rows = s["mask_rows"].tolist() if s["masks"] else None
    shift = torch.arange(32, device=DEV, dtype=torch.int32)
    for i, n in enumerate(s["n"]):
        if s["biases"]:
            a, b = int(s["bias_start"][i]), int(s["bias_start"][i + 1])
            bias = torch.zeros(vocab, dtype=torch.float64, device=DEV)
            bias.index_add_(0, s["bias_tokens"][a:b].long(), s["bias_values"][a:b].double())
        if s["penalties"]:
            c = s["counts"][slots[i]].double().clone()
            words = s["seen"][slots[i], 0]
            prompt = torch.stack([(words >> k) & 1 for k in shift.tolist()], dim=1).reshape(-1)[:vocab].bool()
            r, f, p = (float(s[k][i]) for k in ("repetition", "frequency", "presence"))
        for j in range(n):
            x = out[starts[i] + j]
            if s["penalties"]:
                if j:
                    c[tokens[starts[i] + j]] += 1
                had = c > 0
                x[(prompt | had) & (x > 0)] /= r
                x[(prompt | had) & (x < 0)] *= r
                x -= f * c + p * had
            if s["biases"]:
                x += bias
            if rows is not None and rows[starts[i] + j] >= 0:
                words = s["mask"][rows[starts[i] + j]]
                x[torch.stack([(words >> k) & 1 for k in shift.tolist()], dim=1).reshape(-1)[:vocab] == 0] = -math.inf
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op == "count_tokens":
        return None
    if op == "adjust_logits":
        return _exact_adjust(s)
    if op == "norm_rotary":
        return _exact_norm_turn(s, s["q"], s["q_weight"]), _exact_norm_turn(s, s["k"], s["k_weight"])
    S, hkv, d = s["S"], s["hkv"], s["d"]
    table, kc = s["block_tables"].cpu().tolist(), s["k_cache"]
    start = 0
    if op == "norm_rotary_append":
        q, k = _exact_norm_turn(s, s["q"], s["q_weight"]), _exact_norm_turn(s, s["k_new"], s["k_weight"])
        kc, vc = kc.double(), s["v_cache"].double()
        for i, n in enumerate(s["n"]):
            p = torch.arange(S[i] - n, S[i], device=DEV)
            b = s["block_tables"][i].long()[p // BLOCK]
            kc[b, :, :, p % BLOCK] = k[start:start + n].view(n, hkv, kc.shape[2], kc.shape[4])
            vc[b, :, :, p % BLOCK] = s["v_new"][start:start + n].double()
            start += n
        return q, kc, vc
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    group = s["hq"] // hkv
    for i, n in enumerate(s["n"]):
        b = torch.tensor(table[i][:(S[i] + BLOCK - 1) // BLOCK], device=DEV)
        pos = torch.arange(S[i] - n, S[i], device=DEV).repeat_interleave(group)
        hidden = torch.arange(S[i], device=DEV) > pos[:, None]
        for g in range(hkv):
            # [blocks][D/x][16][x] -> [keys][D], [blocks][D][16] -> [keys][D]
            k = kc[b, g].transpose(1, 2).reshape(-1, d)[:S[i]].double()
            v = s["v_cache"][b, g].transpose(1, 2).reshape(-1, d)[:S[i]].double()
            q = s["q"][start:start + n, g * group:(g + 1) * group].reshape(-1, d).double()
            x = (q @ k.t() / math.sqrt(d)).masked_fill(hidden, -math.inf)
            if s["sink_logits"] is not None:
                last = s["sink_logits"][g * group:(g + 1) * group].double().repeat(n)[:, None]
                x = torch.cat([x, last], dim=1)
            out[start:start + n, g * group:(g + 1) * group] = (torch.softmax(x, dim=1)[:, :S[i]] @ v).view(n, group, d)
        start += n
    return out
