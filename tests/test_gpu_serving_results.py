"""What the tests of the serving calls leave open: every combination of penalties, biases
and masks; each replay of a captured decoding loop against the oracle; and the caches
around the slots that a verify step appends to."""
from __future__ import annotations

import itertools

import numpy as np
import pytest
import torch

import oracle
import paper_2608_24004_amd as av
import workload
from bounded_common import bits
from oracle import serving
from test_gpu_agents_step import CASES as ENGINES
from test_gpu_agents_step import _engine
from test_gpu_logits import _case, _check, _dev

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

PENALTIES = ["".join(p) for k in range(4) for p in itertools.combinations("rfp", k)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("masks", [False, True], ids=["free", "masked"])
@pytest.mark.parametrize("biases", [0, 6])
@pytest.mark.parametrize("penalties", PENALTIES, ids=[p or "none" for p in PENALTIES])
def test_every_combination_of_changes(penalties, biases, masks, dtype):
    n, V = [4, 0, 1, 9], 4133
    x, c, kw = _case(31 + len(penalties), n, V, penalties=penalties, biases=biases, masks=masks, special=True)
    x_t = torch.as_tensor(x).to(workload.torch_dtype(dtype))
    ref, size, touched = serving.adjust_logits(x_t.double().numpy(), c["tokens"], c["q_start"], **kw)
    dev = {k: _dev(v) for k, v in kw.items()}
    logits = x_t.to(DEV)
    got = av.verify_adjust_logits(logits, _dev(c["tokens"]), _dev(c["q_start"]), **dev)
    _check(x_t, got, ref, size, touched, dtype)
    av.verify_adjust_logits(logits, _dev(c["tokens"]), _dev(c["q_start"]), out=logits, **dev)
    np.testing.assert_array_equal(bits(logits), bits(got))


def test_each_replay_of_a_decoding_loop_against_the_oracle():
    n, V = [4, 1, 3, 2], 3001
    x, c, kw = _case(12, n, V, penalties="rfp", biases=5, masks=True)
    B, T = len(n), sum(n)
    dev = {k: _dev(v) for k, v in kw.items()}
    tok, qs = _dev(c["tokens"]), _dev(c["q_start"])
    logits = torch.as_tensor(x, dtype=torch.float32, device=DEV)
    out = torch.empty_like(logits)
    i32 = dict(dtype=torch.int32, device=DEV)
    names = ("argmax_out", "accept_len", "num_emitted", "emitted")
    outs = {k: torch.empty(T if k in ("argmax_out", "emitted") else B, **i32) for k in names}
    ws = torch.empty(av.accept_workspace_size(B, T, V, av.F32), dtype=torch.uint8, device=DEV)

    def step():
        av.verify_adjust_logits(logits, tok, qs, out=out, **dev)
        av.verify_accept(out, tok, qs, workspace=ws, **outs)
        av.verify_count_tokens(dev["counts"], dev["seen"], outs["emitted"], qs, num_tokens=outs["num_emitted"],
                               slots=dev["slots"])

    step()
    torch.cuda.synchronize()
    dev["counts"].copy_(_dev(kw["counts"]))
    dev["seen"].copy_(_dev(kw["seen"]))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    state = dict(kw)
    for replay in range(4):
        logits.normal_(generator=torch.Generator(device=DEV).manual_seed(replay)).mul_(4)
        x_t = logits.cpu()
        g.replay()
        torch.cuda.synchronize()
        ref, size, touched = serving.adjust_logits(x_t.double().numpy(), c["tokens"], c["q_start"], **state)
        _check(x_t, out, ref, size, touched, "f32")
        best = oracle.argmax(out.cpu().numpy(), 0, with_gap=False)
        best = best[0] if isinstance(best, tuple) else best
        want = dict(zip(names, (best,) + tuple(oracle.accept(c["q_start"], c["tokens"], best))))
        for k in names:
            np.testing.assert_array_equal(outs[k].cpu().numpy(), want[k])
        counts, seen = serving.count_tokens(state["counts"], state["seen"], want["emitted"], c["q_start"],
                                            num=want["num_emitted"], slots=kw["slots"])
        np.testing.assert_array_equal(dev["counts"].cpu().numpy(), counts)
        np.testing.assert_array_equal(dev["seen"].cpu().numpy(), seen)
        state.update(counts=counts, seen=seen)
    assert int(state["counts"].sum()) - int(kw["counts"].sum()) >= 4 * B


@pytest.mark.parametrize("dtype,hq,hkv,d", ENGINES)
def test_the_append_writes_its_slots_of_both_caches_alone(dtype, hq, hkv, d):
    e = _engine(dtype, hq, hkv, d, 2)
    for _ in range(2):
        e.before()
        k0, v0 = e.k.clone(), e.v.clone()
        e.first()
        at, slot = e.table.long()[e.req, e.positions.long() // 16], e.positions.long() % 16
        np.testing.assert_array_equal(bits(e.v[at, :, :, slot]), bits(e.qkv[:, hq + hkv:]))
        assert not torch.equal(bits_of(e.k), bits_of(k0)) and not torch.equal(bits_of(e.v), bits_of(v0))
        k, v = e.k.clone(), e.v.clone()
        k[at, :, :, slot], v[at, :, :, slot] = k0[at, :, :, slot], v0[at, :, :, slot]
        assert torch.equal(bits_of(k), bits_of(k0)) and torch.equal(bits_of(v), bits_of(v0))
        e.lm_head()
        e.second()
        e.after()


def bits_of(t):
    return t.view(torch.uint8)
