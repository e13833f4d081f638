"""The operators of a bounded cache together, as a server runs them: append, attend and add up weights, evict when the
budget is passed, and the sliding window over the same cache; against a simulation in 64 bits."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import KL, REL, keep, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


class Stream:
    """Caches on the GPU, and each value head's rows and weights in 64 bits."""

    def __init__(self, B, Hq, Hkv, P, budget, spare, seed=1):
        self.B, self.Hq, self.Hkv, self.P, self.budget = B, Hq, Hkv, P, budget
        self.gen = torch.Generator().manual_seed(seed)
        per = -(-(budget + spare) // P)
        self.E = budget + spare
        self.table = torch.randperm(B * per, generator=self.gen).to(torch.int32).view(B, per).cuda()
        self.v = torch.randn(B * per, Hkv, P, 128, generator=self.gen).to(torch.bfloat16).cuda()
        self.w_r = (torch.randn(Hkv, 128, 128, generator=self.gen) / 128 ** 0.5).to(torch.bfloat16).cuda()
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.weights = torch.zeros(B, Hkv, self.E, device="cuda")
        self.kept = torch.zeros(B, Hkv, budget, dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.shape = kl.make_shape(B, Hq, Hkv, 128, P, B * per, per)
        self.rows = [[torch.zeros(0, 128, dtype=torch.float64) for _ in range(Hkv)] for _ in range(B)]
        self.sums = [[torch.zeros(0, dtype=torch.float64) for _ in range(Hkv)] for _ in range(B)]
        sizes = [f for n in (1, 3, 8, 40) for f in (kl.kl_weights_workspace_size(self.shape, n * B, n, self.E, 0),
                                                    kl.kl_window_workspace_size(self.shape, n * B, n, 64, 4, 0))]
        self.ws = workspace(max(sizes + [kl.kl_evict_workspace_size(self.shape, self.E, budget)]))

    def step(self, n, decay, out, window=0, sinks=0):
        """n new tokens per sequence: (weights' outputs, window's outputs)."""
        B = self.B
        q = torch.randn(B * n, self.Hq, 128, generator=self.gen).to(torch.bfloat16)
        new = torch.randn(B * n, self.Hkv, 128, generator=self.gen).to(torch.bfloat16)
        cu = torch.arange(0, (B + 1) * n, n, dtype=torch.int32, device="cuda")
        self.lens += n
        for b in range(B):                             # (a new token starts without weight)
            L = int(self.lens[b])
            self.weights[b, :, L - n:L] = 0.0
        qd = q.cuda()
        kl.kl_append_v_chunk(self.shape, new.cuda(), self.table, self.lens, cu, B * n, n, self.v, self.err)
        o = torch.full((B * n, self.Hq, 128), math.nan, dtype=out, device="cuda")
        kl.kl_attention_weights(self.shape, qd, self.w_r, self.v, self.table, self.lens, cu, B * n, n, self.weights,
                                self.E, decay, self.weights, 0, o, KL[out], self.ws, self.err)
        w = torch.full_like(o, math.nan)
        if window:
            kl.kl_window_attention(self.shape, qd, self.w_r, self.v, self.table, self.lens, cu, B * n, n, window, sinks,
                                   0, w, KL[out], self.ws, self.err)
        want, want_w = torch.zeros(B * n, self.Hq, 128, dtype=torch.float64), torch.zeros(B * n, self.Hq, 128, dtype=torch.float64)
        G, r = self.Hq // self.Hkv, self.w_r.cpu().double()
        for b in range(B):
            for g in range(self.Hkv):
                rows = torch.cat([self.rows[b][g], new[b * n:(b + 1) * n, g].double()])
                self.rows[b][g], L = rows, rows.shape[0]
                sums = torch.cat([self.sums[b][g], torch.zeros(n, dtype=torch.float64)]) * decay
                qr = torch.einsum("ihk,kj->ihj", q[b * n:(b + 1) * n, g * G:(g + 1) * G].double(), r[g])
                s = torch.einsum("ihd,td->iht", qr, rows) / math.sqrt(128)
                p = torch.arange(L - n, L)[:, None, None]
                t = torch.arange(L)
                a = torch.softmax(s.masked_fill(t > p, -math.inf), -1)
                want[b * n:(b + 1) * n, g * G:(g + 1) * G] = a @ rows
                self.sums[b][g] = sums + a.sum((0, 1))
                if window:
                    a = torch.softmax(s.masked_fill((t > p) | ((t >= sinks) & (t <= p - window)), -math.inf), -1)
                    want_w[b * n:(b + 1) * n, g * G:(g + 1) * G] = a @ rows
        for got, ref in ((o, want), (w, want_w)):
            if torch.isfinite(ref).all() and float(ref.norm()):
                d = got.cpu().double() - ref
                assert float(d.norm()) <= REL[out] * float(ref.norm())
        for b in range(B):
            for g in range(self.Hkv):
                L = self.sums[b][g].numel()
                d = self.weights[b, g, :L].cpu().double() - self.sums[b][g]
                assert float(d.norm()) <= REL[torch.float32] * float(self.sums[b][g].norm())

    def evict(self, sinks, recent):
        before, lens = self.weights.clone(), self.lens.tolist()
        kl.kl_evict(self.shape, self.weights, self.E, self.budget, sinks, recent, self.table, self.lens, self.table,
                    self.v, self.weights, self.kept, self.lens, self.ws, self.err)
        for b, L in enumerate(lens):
            for g in range(self.Hkv):
                ids = keep(before[b, g].tolist(), L, self.budget, sinks, recent)
                assert self.kept[b, g, :len(ids)].tolist() == ids
                self.rows[b][g], self.sums[b][g] = self.rows[b][g][ids], self.sums[b][g][ids]
        assert self.lens.tolist() == [min(L, self.budget) for L in lens]


@pytest.mark.parametrize("Hq,Hkv,P", [(8, 2, 16), (4, 4, 32), (16, 1, 128)])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_a_stream_that_goes_on(Hq, Hkv, P, out):
    s = Stream(3, Hq, Hkv, P, budget=150, spare=40)
    s.step(40, 0.0, out)                               # a prompt, in pieces
    for i in range(3):
        s.step(8, 1.0, out, window=64, sinks=4)
    for i in range(150):
        s.step(1 if i % 5 else 3, 0.96875, out, window=64, sinks=4)
        if int(s.lens.max()) > 180:
            s.evict(4, 20)
    assert int(s.err) == 0
    assert int(s.lens.max()) <= 190


def test_captured_steps():
    """Append, weights, eviction and window in one graph, replayed, against the same calls one by one."""
    def make():
        s = Stream(2, 8, 2, 16, budget=100, spare=60)
        for _ in range(12):
            s.step(8, 1.0, torch.float32)
        return s

    one, two = make(), make()
    q = torch.randn(2, 8, 128, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()
    new = torch.randn(2, 2, 128, generator=torch.Generator().manual_seed(10)).to(torch.bfloat16).cuda()
    cu = torch.arange(3, dtype=torch.int32, device="cuda")

    def step(s, out):
        s.lens += 1
        kl.kl_append_v(s.shape, new, s.table, s.lens - 1, s.v, s.err)
        kl.kl_attention_weights(s.shape, q, s.w_r, s.v, s.table, s.lens, cu, 2, 1, s.weights, s.E, 0.5, s.weights, 0, out[0],
                                kl.KL_FP32, s.ws, s.err)
        kl.kl_evict(s.shape, s.weights, s.E, 100, 4, 10, s.table, s.lens, s.table, s.v, s.weights, s.kept, s.lens, s.ws,
                    s.err)
        kl.kl_window_attention(s.shape, q, s.w_r, s.v, s.table, s.lens, cu, 2, 1, 30, 4, 0, out[1], kl.KL_BF16, s.ws, s.err)

    outs = [[torch.zeros(2, 8, 128, device="cuda"), torch.zeros(2, 8, 128, dtype=torch.bfloat16, device="cuda")] for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(one, outs[0])
    for _ in range(20):
        graph.replay()
        step(two, outs[1])
        torch.cuda.synchronize()
        for a, b in ((outs[0][0], outs[1][0]), (outs[0][1], outs[1][1]), (one.weights, two.weights), (one.v, two.v),
                     (one.lens, two.lens), (one.kept, two.kept)):
            assert torch.equal(a, b)
    assert int(one.err) == int(two.err) == 0 and one.lens.tolist() == [100, 100]


def test_two_streams_with_workspaces_of_their_own():
    sets = [Stream(2, 8, 2, 16, budget=100, spare=60, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(6):
        for s, on in zip(sets, streams):
            with torch.cuda.stream(on):
                s.step(8, 1.0, torch.float32, window=20, sinks=2)
    torch.cuda.synchronize()
    assert all(int(s.err) == 0 for s in sets)
