"""verify_adjust_logits and verify_count_tokens against the oracle."""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
import workload
from bounded_common import bits, q_start_of
from oracle import serving

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _dev(x):
    return None if x is None else torch.as_tensor(x).to(DEV)


def _case(seed, n, V, *, history=200, penalties="rfp", biases=0, masks=False, extra_slots=2, special=False):
    """Numpy inputs: rows of n[i] per request, a state of history tokens per slot."""
    rng = np.random.default_rng(seed)
    B, T = len(n), int(sum(n))
    slots_n = B + extra_slots
    x = rng.standard_normal((T, V)) * 4
    if special and T:
        for v in (np.nan, np.inf, -np.inf, 0.0, -0.0):
            x[rng.integers(T, size=V // 4), rng.integers(V, size=V // 4)] = v
    counts = np.zeros((slots_n, V), dtype=np.int32)
    prompt = np.zeros((slots_n, V), dtype=bool)
    for s in range(slots_n):
        np.add.at(counts[s], (rng.random(history) ** 3 * V).astype(int), 1)
        prompt[s, rng.integers(V, size=history)] = True
    seen = np.stack([serving.words(prompt), serving.words(counts > 0)], axis=1)
    c = dict(tokens=rng.integers(0, V, size=T).astype(np.int32), q_start=q_start_of(n))
    if T > 3:  # drafts that repeat, one outside the vocabulary
        c["tokens"][T // 2:T // 2 + 2] = c["tokens"][T // 2]
        c["tokens"][T // 3] = [V, -1, 2 ** 31 - 1][seed % 3]
    kw = {}
    if penalties:
        kw.update(counts=counts, seen=seen, slots=rng.permutation(slots_n)[:B].astype(np.int32))
        if "r" in penalties:
            kw["repetition"] = (0.7 + rng.random(B)).astype(np.float32)
        if "f" in penalties:
            kw["frequency"] = rng.standard_normal(B).astype(np.float32)
        if "p" in penalties:
            kw["presence"] = rng.standard_normal(B).astype(np.float32)
    if biases:
        m = rng.integers(0, 2 * biases, size=B)
        kw["bias_start"] = q_start_of(m)
        kw["bias_tokens"] = rng.integers(-1, V + 1, size=m.sum()).astype(np.int32)
        if m.sum() > 4:
            kw["bias_tokens"][1:4] = kw["bias_tokens"][0]  # named four times
        kw["bias_values"] = (5 * rng.standard_normal(m.sum())).astype(np.float32)
    if masks:
        allowed = rng.random((5, V)) < np.array([1.0, 0.97, 0.5, 0.01, 0.0])[:, None]
        kw["mask"] = serving.words(allowed)
        kw["mask_rows"] = rng.integers(-1, 6, size=T).astype(np.int32)
    return x, c, kw


def _check(x_t, got, ref, size, touched, dtype):
    """Half a step of the storage type and, in fp32, one of each operand that the oracle
    counts and of the result."""
    with np.errstate(invalid="ignore"):
        tol = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype] * np.abs(ref) + 2.0 ** -24 * (size + np.abs(ref)) * (1 + 2.0 ** -6)
        tol = tol * (1 + 2.0 ** -7)
        g = got.to(torch.float64).cpu().numpy()
        fine = np.isfinite(ref)
        np.testing.assert_array_equal(g[~fine], ref[~fine])
        bad = fine & ~(np.abs(g - ref) <= tol)
    assert not bad.any(), "%d of %d off" % (bad.sum(), bad.size)
    same = ~touched & ~np.isnan(ref)
    np.testing.assert_array_equal(bits(got)[same], bits(x_t)[same])


CASES = [
    # n, V, options
    ([1], 8, dict()),
    ([1], 1, dict(biases=2, masks=True)),
    ([3, 0, 5], 301, dict(biases=3, masks=True, special=True)),
    ([9, 1, 4], 5003, dict(biases=40, masks=True)),
    ([2, 2], 4096, dict(penalties="", masks=True)),
    ([2, 2], 4104, dict(penalties="", biases=600)),
    ([17, 1, 2, 6], 20000, dict(penalties="f", special=True)),
    ([70], 6000, dict(penalties="rp", history=2000, masks=True)),   # rows divided over workgroups
    ([700, 3], 2500, dict(penalties="rfp", biases=4, masks=True)),  # more rows than a workgroup keeps entries of
    ([1] * 40, 2056, dict(biases=5)),
    ([4, 3], 30000, dict(penalties="r", history=0)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,opt", CASES)
def test_adjust_logits(n, V, opt, dtype):
    x, c, kw = _case(V + len(n), n, V, **opt)
    x_t = torch.as_tensor(x).to(workload.torch_dtype(dtype))
    ref, size, touched = serving.adjust_logits(x_t.double().numpy(), c["tokens"], c["q_start"], **kw)
    dev = {k: _dev(v) for k, v in kw.items()}
    before = [v.clone() for v in dev.values()]
    tok, qs = _dev(c["tokens"]), _dev(c["q_start"])
    logits = x_t.to(DEV)
    got = av.verify_adjust_logits(logits, tok, qs, **dev)
    _check(x_t, got, ref, size, touched, dtype)
    np.testing.assert_array_equal(bits(logits), bits(x_t))
    # rows of a wider matrix, 16-byte aligned and not; in place: the same bits
    for pad, off in ((8, 0), (24, 8), (1, 0), (5, 3)):
        wide = torch.full((len(x), V + pad + off), 9.0, dtype=x_t.dtype, device=DEV)
        part = wide[:, off:off + V]
        part.copy_(logits)
        out = torch.full_like(wide, 3.0)
        assert av.verify_adjust_logits(part, tok, qs, out=out[:, off:off + V], **dev) is not None
        np.testing.assert_array_equal(bits(out[:, off:off + V]), bits(got))
        assert (out[:, :off] == 3).all() and (out[:, off + V:] == 3).all()
        av.verify_adjust_logits(part, tok, qs, out=part, **dev)
        np.testing.assert_array_equal(bits(part), bits(got))
        assert (wide[:, :off] == 9).all() and (wide[:, off + V:] == 9).all()
    for a, b in zip(before, dev.values()):
        assert torch.equal(a, b)


def test_slots_outside_the_state_and_rows_behind_the_last_request():
    x, c, kw = _case(3, [3, 2, 4], 999, penalties="rfp")
    kw["slots"] = np.array([-1, 1, 77], dtype=np.int32)
    x = np.concatenate([x, x[:2]])  # two rows of no request
    tokens = np.concatenate([c["tokens"], [5, 6]]).astype(np.int32)
    x_t = torch.as_tensor(x, dtype=torch.bfloat16)
    ref, size, touched = serving.adjust_logits(x_t.double().numpy(), tokens, c["q_start"], **kw)
    out = torch.full(x_t.shape, 3.0, dtype=x_t.dtype, device=DEV)
    av.verify_adjust_logits(x_t.to(DEV), _dev(tokens), _dev(c["q_start"]), out=out, **{k: _dev(v) for k, v in kw.items()})
    _check(x_t[:9], out[:9], ref[:9], size[:9], touched[:9], "bf16")
    assert (out[9:] == 3).all()


def test_a_row_whose_mask_lacks_all_is_minus_infinity_and_accepts_the_first_token():
    V = 1000
    logits = torch.randn((2, V), device=DEV)
    logits[1, 4] = float("nan")
    mask = torch.zeros((1, (V + 31) // 32), dtype=torch.int32, device=DEV)
    rows = torch.zeros(2, dtype=torch.int32, device=DEV)
    tok, qs = torch.tensor([1, 2], dtype=torch.int32, device=DEV), torch.tensor([0, 2], dtype=torch.int32, device=DEV)
    got = av.verify_adjust_logits(logits, tok, qs, mask=mask, mask_rows=rows)
    assert (got == -float("inf")).all()
    assert av.verify_accept(got, tok, qs)[3].tolist() == [0, 0]


@pytest.mark.parametrize("V", [1, 31, 301, 5003, 40000])
@pytest.mark.parametrize("prompt", [False, True])
def test_count_tokens(V, prompt):
    rng = np.random.default_rng(V)
    n = [0, 1, 5, 700, 3, 3000]
    start = q_start_of(n)
    tokens = (rng.random(start[-1] + 3) ** 4 * (V + 2)).astype(np.int32) - 1  # -1 and V among them
    num = np.array([4, 1, 0, 650, 9, 2999], dtype=np.int32)
    slots = np.array([0, 2, 5, 2, 9, 1], dtype=np.int32)  # slot 2 twice, slot 9 not there
    counts = rng.integers(0, 3, size=(6, V)).astype(np.int32)
    seen = np.stack([serving.words(rng.random((6, V)) < 0.3), serving.words(counts > 0)], axis=1)
    for kw in (dict(num=num, slots=slots), dict(num=None, slots=slots), dict(num=num, slots=None)):
        want = serving.count_tokens(counts, seen, tokens, start, prompt=prompt, **kw)
        c, s = _dev(counts), _dev(seen)
        av.verify_count_tokens(c, s, _dev(tokens), _dev(start), num_tokens=_dev(kw["num"]), slots=_dev(kw["slots"]),
                               prompt=prompt)
        np.testing.assert_array_equal(c.cpu().numpy(), want[0])
        np.testing.assert_array_equal(s.cpu().numpy(), want[1])


def test_a_total_near_the_largest_bounds_the_requests_alone():
    """total_tokens and total_q only clamp where requests begin and end: no memory behind
    the last request is touched, and the launch is as large as any."""
    V, B = 1000, 2
    counts = torch.zeros(B, V, dtype=torch.int32, device=DEV)
    seen = torch.zeros(B, 2, (V + 31) // 32, dtype=torch.int32, device=DEV)
    tokens = torch.tensor([7, 7, 999, 3], dtype=torch.int32, device=DEV)
    start = torch.tensor([0, 3, 4], dtype=torch.int32, device=DEV)
    rc = av.library().verify_count_tokens(B, 2 ** 31 - 1, V, B, tokens.data_ptr(), start.data_ptr(), None, None, 0,
                                          counts.data_ptr(), seen.data_ptr(), None)
    assert rc == av.OK
    torch.cuda.synchronize()
    want = torch.zeros(B, V, dtype=torch.int32)
    want[0, 7], want[0, 999], want[1, 3] = 2, 1, 1
    assert torch.equal(counts.cpu(), want)
    x = torch.randn(4, V, device=DEV)
    out = torch.full_like(x, 5.0)
    pen = torch.ones(B, device=DEV)
    p = av.AdjustParams(presence=pen.data_ptr(), counts=counts.data_ptr(), seen=seen.data_ptr(), num_slots=B)
    rc = av.library().verify_adjust_logits(B, 2 ** 30 - 1, V, 0, av.F32, x.data_ptr(), tokens.data_ptr(),
                                           start.data_ptr(), ctypes.byref(p), out.data_ptr(), 0, None)
    assert rc == av.OK
    torch.cuda.synchronize()
    got, y = out.cpu(), x.cpu()
    for row, had in enumerate([{7, 999}, {7, 999}, {7, 999}, {3}]):
        for v in had:
            y[row, v] -= 1
    assert torch.equal(got, y)


def test_the_calls_of_decoding_captured_and_replayed():
    """Adjust, accept, count, as a decoding loop captures them: each replay reads what
    the one before has counted."""
    n, V = [4, 1, 3], 3001
    x, c, kw = _case(8, n, V, penalties="rfp", masks=True)
    kw["mask_rows"][:] = -1  # every token may follow, so that none is -inf
    dev = {k: _dev(v) for k, v in kw.items()}
    tok, qs, logits = _dev(c["tokens"]), _dev(c["q_start"]), torch.as_tensor(x, dtype=torch.float32, device=DEV)
    out = torch.empty_like(logits)
    B, T = len(n), sum(n)
    i32 = dict(dtype=torch.int32, device=DEV)
    outs = dict(argmax_out=torch.empty(T, **i32), accept_len=torch.empty(B, **i32), num_emitted=torch.empty(B, **i32),
                emitted=torch.empty(T, **i32))
    ws = torch.empty(av.accept_workspace_size(B, T, V, av.F32), dtype=torch.uint8, device=DEV)

    def step(counts, seen, out, outs):
        av.verify_adjust_logits(logits, tok, qs, out=out, **{**dev, "counts": counts, "seen": seen})
        av.verify_accept(out, tok, qs, workspace=ws, **outs)
        av.verify_count_tokens(counts, seen, outs["emitted"], qs, num_tokens=outs["num_emitted"], slots=dev["slots"])

    counts, seen = dev["counts"].clone(), dev["seen"].clone()
    step(counts, seen, out, outs)
    torch.cuda.synchronize()
    counts.copy_(dev["counts"])
    seen.copy_(dev["seen"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(counts, seen, out, outs)
    mine = dev["counts"].clone(), dev["seen"].clone()
    out1, outs1 = torch.empty_like(out), {k: torch.empty_like(v) for k, v in outs.items()}
    emitted = []
    for _ in range(4):
        g.replay()
        step(*mine, out1, outs1)
        torch.cuda.synchronize()
        assert torch.equal(counts, mine[0]) and torch.equal(seen, mine[1])
        np.testing.assert_array_equal(bits(out), bits(out1))
        emitted.append(outs["emitted"].tolist())
    ref, size, touched = serving.adjust_logits(logits.double().cpu().numpy(), c["tokens"], c["q_start"],
                                               **{**kw, "counts": dev["counts"].cpu().numpy()})
    assert int(counts.sum()) - int(dev["counts"].sum()) >= 4 * B
