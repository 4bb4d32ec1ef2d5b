"""The calls of a bounded cache at their edges: rows and keys that are not finite,
beside places without a row."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2608_24004_amd as av
import workload
from bounded_common import Cache, q_start_of
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
