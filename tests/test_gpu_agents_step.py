"""The calls of a verify step of agents that share their instructions, one after the
other as a serving engine makes them: norms, rotation and append; attention with the
common prefix; logits changed by penalties, biases and a grammar; greedy acceptance;
counts of what stands.  Every call's result is checked against the oracle on the inputs
that the calls before it left, and a captured step against the eager one, bit for bit."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import paper_2608_24004_amd as av
import workload
from bounded_common import bits, q_start_of
from oracle import serving
from shared_common import SharedBatch
from test_gpu_logits import _check
from test_gpu_norm_rotary import _close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
V = 3001
EPS = 1e-6


class Engine:
    """Requests that decode drafts of fixed lengths; all state on the GPU.  Row j's query,
    key and value depend on its token and position alone."""

    def __init__(self, dtype, hq, hkv, d, groups, S, n, steps):
        self.b = b = SharedBatch(21, groups, S, n, hq=hq, hkv=hkv, d=d, dtype=dtype, sinks=True)
        self.n, self.dtype = n, dtype
        B, T = len(n), sum(n)
        room = max(S) + steps * max(n)
        g = torch.Generator(device=DEV).manual_seed(5)
        q, self.k, self.v, table, self.seq_lens, self.q_start, self.gs, self.pl = b.to(DEV)
        # blocks for the keys to come
        extra = steps * max(n) // 16 + 2
        nb, have = self.k.shape[0], table.shape[1]
        grown = torch.full((B, have + extra), -1, dtype=torch.int32, device=DEV)
        grown[:, :have] = table
        for i in range(B):
            used = -(-S[i] // 16)
            grown[i, used:used + extra] = torch.arange(nb + i * extra, nb + (i + 1) * extra, dtype=torch.int32, device=DEV)
        self.table = grown
        more = lambda c: torch.cat([c, torch.full((B * extra,) + c.shape[1:], float("nan"), dtype=c.dtype, device=DEV)])
        self.k, self.v = more(self.k), more(self.v)
        self.bounds = dict(max_q_len=max(n), max_seq_len=room, max_prefix_len=int(b.prefix.max()))
        dt = q.dtype
        self.embed = torch.randn((V, (hq + 2 * hkv) * d), generator=g, device=DEV).to(dt)
        self.head = torch.randn((hq * d, V), generator=g, device=DEV) / 4
        self.weights = [torch.rand((d,), generator=g, device=DEV) + 0.5 for _ in range(2)]
        self.freq = torch.as_tensor(10000.0 ** (-np.arange(d // 2) / (d // 2)), device=DEV)
        self.tokens = torch.randint(0, V, (T,), generator=g, device=DEV).to(torch.int32)
        self.counts = torch.zeros((B, V), dtype=torch.int32, device=DEV)
        self.seen = torch.zeros((B, 2, (V + 31) // 32), dtype=torch.int32, device=DEV)
        prompts = torch.randint(0, V, (B * 40,), generator=g, device=DEV).to(torch.int32)
        av.verify_count_tokens(self.counts, self.seen, prompts, torch.arange(0, B * 40 + 1, 40, dtype=torch.int32, device=DEV),
                               prompt=True)
        self.par = dict(repetition=torch.full((B,), 1.3, device=DEV), frequency=torch.full((B,), 0.4, device=DEV),
                        presence=torch.full((B,), 0.2, device=DEV))
        rng = np.random.default_rng(3)
        self.mask = torch.as_tensor(serving.words(rng.random((4, V)) < np.array([1, 0.5, 0.1, 0.01])[:, None])).to(DEV)
        self.mask_rows = torch.as_tensor(rng.integers(-1, 4, size=T).astype(np.int32)).to(DEV)
        self.req = torch.repeat_interleave(torch.arange(B, device=DEV), torch.as_tensor(n, device=DEV))
        self.j = torch.arange(T, device=DEV) - self.q_start.long()[self.req]
        self.positions = torch.empty((T,), dtype=torch.int32, device=DEV)
        self.qkv = torch.empty((T, (hq + 2 * hkv), d), dtype=dt, device=DEV)
        self.q_out, self.out = torch.empty((T, hq, d), dtype=dt, device=DEV), torch.empty((T, hq, d), dtype=dt, device=DEV)
        self.logits, self.changed = (torch.empty((T, V), device=DEV) for _ in range(2))
        i32 = dict(dtype=torch.int32, device=DEV)
        self.accepted = dict(argmax_out=torch.empty(T, **i32), accept_len=torch.empty(B, **i32),
                             num_emitted=torch.empty(B, **i32), emitted=torch.empty(T, **i32))
        self.ws = torch.empty(av.attention_shared_workspace_size(q, self.k, self.table, num_groups=len(groups), **self.bounds),
                              dtype=torch.uint8, device=DEV)
        self.accept_ws = torch.empty(av.accept_workspace_size(B, T, V, av.F32), dtype=torch.uint8, device=DEV)
        self.hq, self.hkv, self.d = hq, hkv, d

    def before(self):
        """What a model's other layers would do, by torch."""
        n = torch.as_tensor(self.n, device=DEV)
        self.positions.copy_((self.seq_lens - n)[self.req] + self.j)
        self.qkv.copy_(self.embed[self.tokens.long()].view(self.qkv.shape))

    def first(self):
        q, k, v = self.qkv.split([self.hq, self.hkv, self.hkv], dim=1)
        av.verify_norm_rotary_append(q, k, v, self.positions, self.freq, self.k, self.v, self.table, self.seq_lens,
                                     self.q_start, q_weight=self.weights[0], k_weight=self.weights[1], eps=EPS,
                                     q_out=self.q_out)
        av.verify_attention_shared(self.q_out, self.k, self.v, self.table, self.seq_lens, self.q_start, self.gs, self.pl,
                                   sinks=self.b.sinks_dev, out=self.out, workspace=self.ws, **self.bounds)

    def lm_head(self):
        torch.mm(self.out.float().view(self.out.shape[0], -1), self.head, out=self.logits)

    def second(self):
        av.verify_adjust_logits(self.logits, self.tokens, self.q_start, counts=self.counts, seen=self.seen, mask=self.mask,
                                mask_rows=self.mask_rows, out=self.changed, **self.par)
        av.verify_accept(self.changed, self.tokens, self.q_start, workspace=self.accept_ws, **self.accepted)
        av.verify_count_tokens(self.counts, self.seen, self.accepted["emitted"], self.q_start,
                               num_tokens=self.accepted["num_emitted"])

    def after(self):
        """The emitted tokens stand; the next drafts are what the rows said, and more."""
        m = self.accepted["num_emitted"]
        self.seq_lens.add_(m)
        last = self.accepted["emitted"][(self.q_start[:-1] + m - 1).long()]
        guess = (self.accepted["argmax_out"] * 7 + 3) % V
        self.tokens.copy_(torch.where(self.j == 0, last[self.req], guess))


CASES = [("bf16", 8, 2, 128), ("f32", 4, 2, 64)]
BATCH = dict(groups=[(3, 200), (2, 70)], S=[210, 230, 204, 90, 75, 40], n=[4, 1, 3, 5, 2, 4])


def _engine(dtype, hq, hkv, d, steps):
    e = Engine(dtype, hq, hkv, d, steps=steps, **BATCH)
    e.b.sinks_dev = e.b.sinks.to(DEV)
    return e


@pytest.mark.parametrize("dtype,hq,hkv,d", CASES)
def test_steps_against_the_oracle(dtype, hq, hkv, d):
    e = _engine(dtype, hq, hkv, d, 3)
    qs = q_start_of(e.n)
    for step in range(3):
        e.before()
        k0, v0 = e.k.clone(), e.v.clone()
        counts0, seen0 = e.counts.cpu().numpy(), e.seen.cpu().numpy()
        e.first()
        x = e.qkv.to(torch.float64).cpu().numpy()
        _close(e.q_out, x[:, :hq], e.weights[0].double().cpu().numpy(), e.positions.cpu().numpy()[None],
               e.freq.cpu().numpy(), [0] * (d // 2), False, 1.0, dtype)
        # what was appended, read back row by row, and nothing else changed
        at = e.table.long()[e.req, e.positions.long() // 16]
        back = e.k[at, :, :, e.positions.long() % 16].reshape(len(x), hkv, d)
        _close(back, x[:, hq:hq + hkv], e.weights[1].double().cpu().numpy(), e.positions.cpu().numpy()[None],
               e.freq.cpu().numpy(), [0] * (d // 2), False, 1.0, dtype)
        np.testing.assert_array_equal(bits(e.v[at, :, :, e.positions.long() % 16]), bits(e.qkv[:, hq + hkv:]))
        e.k[at, :, :, e.positions.long() % 16], kept = k0[at, :, :, e.positions.long() % 16], e.k.clone()
        np.testing.assert_array_equal(bits(e.k), bits(k0))
        e.k.copy_(kept)
        # the attention, over the caches as they are now
        b = e.b
        b.q, b.k, b.v, b.table = e.q_out.cpu(), e.k.cpu(), e.v.cpu(), e.table.cpu().numpy()
        b.S, b.n = e.seq_lens.cpu().numpy(), np.asarray(e.n)
        b.check(e.out, "step %d" % step)
        e.lm_head()
        e.second()
        tokens = e.tokens.cpu().numpy()
        ref, size, touched = serving.adjust_logits(
            e.logits.double().cpu().numpy(), tokens, qs, counts=counts0, seen=seen0, mask=e.mask.cpu().numpy(),
            mask_rows=e.mask_rows.cpu().numpy(), **{k: v.cpu().numpy() for k, v in e.par.items()})
        _check(e.logits, e.changed, ref, size, touched, "f32")
        best = oracle.argmax(e.changed.cpu().numpy(), 0, with_gap=False)
        best = best[0] if isinstance(best, tuple) else best
        acc, num, emitted = oracle.accept(qs, tokens, best)
        for got, want in zip((e.accepted[k] for k in ("argmax_out", "accept_len", "num_emitted", "emitted")),
                             (best, acc, num, emitted)):
            np.testing.assert_array_equal(got.cpu().numpy(), want)
        c, s = serving.count_tokens(counts0, seen0, emitted, qs, num=num)
        np.testing.assert_array_equal(e.counts.cpu().numpy(), c)
        np.testing.assert_array_equal(e.seen.cpu().numpy(), s)
        e.after()


@pytest.mark.parametrize("dtype,hq,hkv,d", CASES)
def test_a_captured_step_is_the_eager_one(dtype, hq, hkv, d):
    eager, graphed = _engine(dtype, hq, hkv, d, 6), _engine(dtype, hq, hkv, d, 6)
    graphed.before()
    graphed.first()
    graphed.second()
    torch.cuda.synchronize()
    fresh = _engine(dtype, hq, hkv, d, 6)
    for name in ("k", "v", "counts", "seen", "seq_lens", "tokens"):
        getattr(graphed, name).copy_(getattr(fresh, name))
    graphs = []
    for part in (graphed.first, graphed.second):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            part()
        graphs.append(g)
    for step in range(5):
        for e in (eager, graphed):
            e.before()
            e.first() if e is eager else graphs[0].replay()
            e.lm_head()
            e.second() if e is eager else graphs[1].replay()
            e.after()
            torch.cuda.synchronize()
        for name in ("q_out", "out", "changed", "k", "v", "counts", "seen", "seq_lens", "tokens"):
            np.testing.assert_array_equal(bits(getattr(eager, name)), bits(getattr(graphed, name)),
                                          err_msg="step %d %s" % (step, name))
    assert int(eager.counts.sum()) >= 5 * len(BATCH["n"])
