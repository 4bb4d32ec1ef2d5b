"""The calls of a bounded cache at their edges: rows and keys that are not finite,
beside places without a row; two streams at once; a kept workspace, a given scale and
checked descriptors."""
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


def _dev(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype, device=DEV)


def _agree(w, rw, tol):
    """Weights within tol of rw, NaN exactly where rw is."""
    w = w.double().cpu().numpy()
    none = np.isnan(rw)
    np.testing.assert_array_equal(np.isnan(w), none)
    assert (np.abs(w - rw)[~none] <= tol[~none]).all()


# (rows that fill their last tile in part: in a tile of 16 rows, the rows of one request)
PROMPTS = [(60, 60, 60, 64, "bf16"), (100, 60, 60, 64, "bf16"), (70, 60, 60, 128, "f32"), (400, 300, 300, 128, "bf16"),
           (100, 60, 2, 128, "bf16")]  # the last announces fewer rows than it has


@pytest.mark.parametrize("S,n,max_q_len,d,dtype", PROMPTS)
def test_a_row_that_is_not_finite_reaches_the_keys_it_sees(S, n, max_q_len, d, dtype):
    """The first row's query holds a NaN: its keys' weights are NaN and no others."""
    rng = np.random.default_rng(S)
    c = Cache(rng, [S], hkv=1, d=d, dtype=dtype)
    q = torch.as_tensor(rng.standard_normal((n, 1, d))).to(workload.torch_dtype(dtype))
    q[0, 0, 7] = float("nan")
    kc, _, w, o, bt, sl = c.to(DEV)
    av.verify_key_weights(q.to(DEV), kc, w, o, bt, sl, _dev(q_start_of([n])), max_q_len=max_q_len, max_seq_len=S)
    k, _, w0, o0 = c.numpy()
    rw, _, tol = bounded.key_weights(q.double().numpy(), k, w0, o0, c.block_tables, [S], q_start_of([n]))
    line = np.concatenate([rw[b, 0] for b in c.block_tables[0]])
    assert np.isnan(line[:S - n + 1]).all() and np.isfinite(line[S - n + 1:S]).all()
    _agree(w, rw, tol)


@pytest.mark.parametrize("S,n,max_q_len,d,dtype", PROMPTS)
def test_an_infinite_key_that_scores_minus_infinity_weighs_nothing(S, n, max_q_len, d, dtype):
    """... in a prompt whose first rows, which do not see the key, have the other sign."""
    rng = np.random.default_rng(S + 1)
    c = Cache(rng, [S], hkv=1, d=d, dtype=dtype)
    key = S - n + 5
    at = (int(c.block_tables[0, key // 16]), 0, 0, key % 16, 0)
    q = torch.as_tensor(rng.standard_normal((n, 1, d))).to(workload.torch_dtype(dtype))
    q[:5, 0, 0], q[5:, 0, 0] = 1.0, -1.0
    # the tolerance, and the ordinals, of the same call with a finite key there
    k, _, w0, o0 = c.numpy()
    k[at] = 1.0
    _, _, tol = bounded.key_weights(q.double().numpy(), k, w0, o0, c.block_tables, [S], q_start_of([n]))
    k[at] = np.inf
    keys = np.stack([k[c.block_tables[0, t // 16], 0, :, t % 16].reshape(d) for t in range(S)])
    rw = w0.copy()
    rw[c.block_tables[0, :(S + 15) // 16], 0] = np.nan
    line = np.array([w0[c.block_tables[0, t // 16], 0, t % 16] if t < S - n else 0.0 for t in range(S)])
    for j in range(n):
        s = keys[:S - n + j + 1] @ q[j, 0].double().numpy() / np.sqrt(d)
        p = np.exp(s - s.max())
        line[:len(s)] += p / p.sum()
    assert np.isfinite(line).all() and line[key] == 0
    for t in range(S):
        rw[c.block_tables[0, t // 16], 0, t % 16] = line[t]
    c.k[at] = float("inf")
    kc, _, w, o, bt, sl = c.to(DEV)
    av.verify_key_weights(q.to(DEV), kc, w, o, bt, sl, _dev(q_start_of([n])), max_q_len=max_q_len, max_seq_len=S)
    _agree(w, rw, tol)


class _Session:
    """One request batch's calls, on copies that are all made beforehand."""

    def __init__(self, seed, S, n, d, copies):
        rng = np.random.default_rng(seed)
        self.c = Cache(rng, S, hkv=2, d=d, dtype="bf16", lost=[50] * len(S))
        self.q, self.k, self.v = (torch.as_tensor(rng.standard_normal((sum(n), h, d))).to(DEV, torch.bfloat16) for h in (8, 2, 2))
        self.pos = _dev(rng.integers(0, 5000, size=(1, sum(n))))
        self.freq = _dev(10000.0 ** (-np.arange(d // 2) / (d // 2)), torch.float64)
        self.qs, self.tokens = _dev(q_start_of(n)), _dev(self.c.tokens)
        self.bounds = dict(max_q_len=max(n), max_seq_len=max(S))
        self.copies = [self.c.to(DEV) for _ in range(copies)]
        # a long cache's weights, whose plan takes a workspace
        self.long = (_dev(rng.exponential(size=(2500, 2, 16)), torch.float32), None,
                     _dev(rng.permutation(2500).reshape(2, 1250)), _dev([20000, 18000 - seed]))

    def run(self, stream):
        kc, vc, w, o, bt, sl = self.copies.pop()
        q = av.verify_rotary_append(self.q, self.k, self.v, self.pos, self.freq, kc, vc, bt, sl, self.qs, stream=stream)
        av.verify_key_weights(q, kc, w, o, bt, sl, self.qs, num_tokens=self.tokens, stream=stream, **self.bounds)
        src, lens = av.verify_evict_plan(w, o, bt, sl, max_keys=128, max_seq_len=self.bounds["max_seq_len"],
                                         num_tokens=self.tokens, stream=stream)
        av.verify_kv_compact(kc, vc, bt, src, lens, key_weights=w, key_order=o, stream=stream)
        far, far_lens = av.verify_evict_plan(*self.long, max_keys=6000, max_seq_len=20000, stream=stream)
        return [q, kc, vc, w, o, src, lens, far, far_lens]


def test_two_streams_at_the_same_time():
    """Calls on two streams with nothing to order them, on different inputs, whose
    workspaces and outputs the binding makes: each as alone."""
    here, there = _Session(1, [700, 400], [300, 20], 64, 5), _Session(2, [900, 350, 40], [9, 3, 9], 128, 5)
    side = torch.cuda.Stream()
    busy = torch.zeros((8192, 8192), dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    want = [[bits(t) for t in x.run(None)] for x in (here, there)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        first = busy @ busy  # both streams have a queue before the calls begin
    second = busy @ busy
    got = [[], []]
    for _ in range(4):
        got[1].append(there.run(side))
        got[0].append(here.run(None))
    torch.cuda.synchronize()
    for runs, ref in zip(got, want):
        for out in runs:
            for a, b in zip(out, ref):
                np.testing.assert_array_equal(bits(a), b)
    del first, second


def test_a_kept_workspace_serves_a_request_with_more_rows_than_announced():
    """The workspace of 32 requests of nine rows, for one of 287: the same bits as in
    one of its own, and nothing behind it is written."""
    rng = np.random.default_rng(3)
    c = Cache(rng, [600], hkv=2, d=128, dtype="bf16")
    q = torch.as_tensor(rng.standard_normal((288, 8, 128))).to(DEV, torch.bfloat16)
    kc, _, w0, o0, bt, sl = c.to(DEV)
    kw = dict(max_q_len=9, max_seq_len=600)
    size = av.key_weights_workspace_size(q, kc, bt.expand(32, -1).contiguous(), **kw)
    buf = torch.full((size + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    out = []
    for ws in (None, buf[:size]):
        w, o = w0.clone(), o0.clone()
        av.verify_key_weights(q[:287], kc, w, o, bt, sl, _dev([0, 287]), workspace=ws, **kw)
        out.append((bits(w), bits(o)))
    assert (buf[size:] == 0xFF).all()
    for a, b in zip(*out):
        np.testing.assert_array_equal(a, b)


@pytest.mark.parametrize("n,dtype", [([1, 1], "bf16"), ([9, 3], "bf16"), ([300, 20], "bf16"), ([9, 3], "f32")])
def test_key_weights_with_a_scale(n, dtype):
    rng = np.random.default_rng(n[0])
    S = [700, 90]
    c = Cache(rng, S, hkv=2, d=64, dtype=dtype)
    q = torch.as_tensor(rng.standard_normal((sum(n), 6, 64))).to(workload.torch_dtype(dtype))
    kc, _, w, o, bt, sl = c.to(DEV)
    av.verify_key_weights(q.to(DEV), kc, w, o, bt, sl, _dev(q_start_of(n)), max_q_len=max(n), max_seq_len=700, scale=0.4)
    k, _, w0, o0 = c.numpy()
    rw, ro, tol = bounded.key_weights(q.double().numpy(), k, w0, o0, c.block_tables, S, q_start_of(n), scale=0.4)
    _agree(w, rw, tol)
    np.testing.assert_array_equal(o.cpu().numpy(), ro)


def test_checked_descriptors():
    """check=True: a good batch gives the same bits, a bad one is refused with nothing
    written."""
    rng = np.random.default_rng(5)
    S, n = [100, 40], [9, 3]
    c = Cache(rng, S, hkv=2, d=64, dtype="bf16")
    q, k, v = (torch.as_tensor(rng.standard_normal((12, h, 64))).to(DEV, torch.bfloat16) for h in (4, 2, 2))
    pos, freq = _dev(np.arange(12)[None]), _dev(1.0 / (np.arange(32) + 1.0), torch.float64)

    def calls(check, lens=None, starts=None, table=None):
        kc, vc, w, o, bt, sl = c.to(DEV)
        bt, sl = bt if table is None else _dev(table), sl if lens is None else _dev(lens)
        qs = _dev(q_start_of(n) if starts is None else starts)
        errors = 0
        for call in (lambda: av.verify_rotary_append(q, k, v, pos, freq, kc, vc, bt, sl, qs, check=check),
                     lambda: av.verify_key_weights(q, kc, w, o, bt, sl, qs, max_q_len=9, max_seq_len=100, check=check)):
            try:
                call()
            except av.BatchError:
                errors += 1
        return errors, [bits(t) for t in (kc, vc, w, o)]

    none, plain = calls(False)
    good, same = calls(True)
    assert none == good == 0
    for a, b in zip(plain, same):
        np.testing.assert_array_equal(a, b)
    table = c.block_tables.copy()
    table[0, 6] = c.nb  # the block of the first request's new keys
    for kw in (dict(lens=[100, 2]), dict(starts=[0, 9, 13]), dict(starts=[0, -1, 12]), dict(table=table)):
        bad, left = calls(True, **kw)
        assert bad == 2, kw
        for a, b in zip(left, (bits(t) for t in (c.k, c.v, c.w, c.o))):
            np.testing.assert_array_equal(a, b)
