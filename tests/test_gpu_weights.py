"""kl_attention_weights against its definition in 64 bits: outputs and the weights added up, head layouts, lengths,
rows, decay, strides, in place, rows that are not finite."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import attention, close, inputs, on, shape_of, weigh, workspace

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def olds(x, stride, seed=3):
    """Weights so far, of everything but the new tokens; beyond the sequences something that must stay."""
    Hkv = x["v_cache"].shape[1]
    gen = torch.Generator().manual_seed(seed)
    w = torch.rand(len(x["news"]), Hkv, stride, generator=gen) ** 4
    t = torch.arange(stride)
    before = torch.tensor([L - n for L, n in zip(x["seq_lens"].tolist(), x["news"])])[:, None, None]
    w = torch.where(t < before, w, 0.0)
    return torch.where(t < x["seq_lens"][:, None, None], w, math.nan)


def check(x, decay, stride=None, types=TYPES, in_place=False, **kw):
    g = on(x)
    lens = x["seq_lens"].tolist()
    old = olds(x, stride or max(lens)).cuda()
    want, added = attention(g, scale=kw.get("scale") or None, composed=kw.get("composed", False))
    for dtype in types:
        mine = old.clone()
        out, new = weigh(g, mine, decay, dtype, new=mine if in_place else None, **kw)
        if out.numel():
            close(out, want, dtype)
        for b, L in enumerate(lens):
            w = decay * torch.nan_to_num(old[b, :, :L].double()) + added[b, :, :L]
            if L:
                close(new[b, :, :L], w)
            rest = new[b, :, L:]
            assert torch.isnan(rest).all() if in_place else (rest == -7.0).all()
        if decay == 0.0 and not in_place:
            assert torch.allclose(new[0, :, :lens[0]].sum(-1),
                                  torch.tensor(float(x["news"][0] * x["q"].shape[1] // x["v_cache"].shape[1]),
                                               device="cuda"), rtol=1e-5)


@pytest.mark.parametrize("L", [1, 2, 63, 64, 65, 127, 128, 129, 700])
@pytest.mark.parametrize("decay", [0.0, 0.9375, 1.0])
def test_lengths(L, decay):
    check(inputs((L, max(L - 1, 1), 0), (1, 1, 0)), decay)


@pytest.mark.parametrize("n", [1, 2, 3, 8, 16, 17, 64, 128])
@pytest.mark.parametrize("committed", [0, 1, 100, 128, 700])
def test_rows(n, committed):
    check(inputs((committed + n, committed + 1, 40), (n, 1, 0)), 0.5)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (12, 2), (28, 4), (32, 1), (64, 8), (40, 2), (128, 1)])
@pytest.mark.parametrize("per_q", [False, True])
def test_head_layouts(Hq, Hkv, per_q):
    for news in ((1, 1, 0), (5, 1, 2)):
        check(inputs((333, 40, 200), news, Hq, Hkv, seed=Hq, wr_per_query_head=per_q), 1.0)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
def test_pages_and_splits(P, splits):
    for news in ((1, 1, 1), (5, 2, 3)):
        check(inputs((1500, 131, 700), news, 16, 2, P), 0.96875, splits=splits)


@pytest.mark.parametrize("stride", [1500, 1501, 1600, 5003])
def test_strides_and_in_place(stride):
    x = inputs((1500, 131, 700), (1, 2, 3), 16, 2)
    check(x, 0.5, stride)
    check(x, 0.5, stride, in_place=True)


def test_scale_composed_queries_and_a_loose_bound():
    x = inputs((300, 77), (3, 1))
    check(x, 1.0, scale=0.2)
    check(x, 1.0, composed=True)
    check(x, 1.0, max_q=100)


def test_decay_0_reads_no_old_weights():
    x = inputs((300, 77), (3, 1))
    g = on(x)
    old = torch.full((2, 2, 300), math.nan, device="cuda")
    _, new = weigh(g, old, 0.0)
    close(new[0], attention(g)[1][0])
    sh, ws = shape_of(g), workspace(kl.kl_weights_workspace_size(shape_of(g), 4, 3, 300, 0))
    out = torch.empty(g["q"].shape, device="cuda")
    again = torch.full_like(new, -7.0)
    kl.kl_attention_weights(sh, g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"], 4, 3, None,
                            300, 0.0, again, 0, out, kl.KL_FP32, ws)
    assert torch.equal(again, new)


def test_pieces_of_a_chunk_add_up():
    """70 new tokens in one call, and in calls of 40 and 30 with lengths of their own."""
    x = inputs((500, 300), (70, 70))
    g = on(x)
    old = torch.nan_to_num(olds(x, 500)).cuda()
    _, one = weigh(g, old, 0.5)
    a, b = dict(g), dict(g)
    a.update(q=torch.cat([g["q"][:40], g["q"][70:110]]), cu_q=torch.tensor([0, 40, 80], dtype=torch.int32).cuda(),
             news=[40, 40], seq_lens=g["seq_lens"] - 30)
    b.update(q=torch.cat([g["q"][40:70], g["q"][110:]]), cu_q=torch.tensor([0, 30, 60], dtype=torch.int32).cuda(),
             news=[30, 30])
    _, w = weigh(a, old, 0.5, new=old.clone())
    _, w = weigh(b, w, 1.0, new=w)
    close(w[0], one[0].double())
    close(w[1, :, :300], one[1, :, :300].double())


def test_bad_lengths_are_reported_and_left():
    x = inputs((300, 200, 100), (2, 2, 2))
    g = on(x)
    old = torch.nan_to_num(olds(x, 300)).cuda()
    want, added = attention(g)
    for L in (-1, 1, 301, 1 << 29):
        g["seq_lens"][1] = L
        out, new = weigh(g, old, 1.0, flags=kl.KL_FLAG_BAD_LENGTH)
        assert torch.isnan(out[2:4]).all() and (new[1] == -7.0).all()
        close(out[:2], want[:2])
        close(new[2, :, :100], old[2, :, :100].double() + added[2, :, :100])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_not_finite(bad):
    """Behind the sequence: nothing; a new token's row: the positions that see it."""
    x = inputs((200, 100), (3, 2), 8, 2)
    for b, L in enumerate((200, 100)):
        for t in range(L, -(-L // 16) * 16):
            x["v_cache"][int(x["block_table"][b, t // 16]), :, t % 16] = bad
    check(x, 1.0)
    x["v_cache"][int(x["block_table"][0, 198 // 16]), :, 198 % 16, 7] = math.nan
    out, new = weigh(on(x), olds(x, 200).cuda(), 1.0)
    want = attention(on(x))[0]
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    close(out[0], want[0])
    close(out[3:], want[3:])
    assert torch.isnan(new[0]).all() and not torch.isnan(new[1, :, :100]).any()


def test_a_workspace_shared_with_a_graph_and_the_same_sums_on_every_run():
    sets = [on(inputs((1500, 40, 800), n, 16, 2, seed=i)) for i, n in enumerate(((1, 1, 1), (3, 2, 4), (64, 1, 30)))]
    old = torch.rand(3, 2, 1500, device="cuda")
    ws = workspace(max(kl.kl_weights_workspace_size(shape_of(g), g["q"].shape[0], max(g["news"]), 1500, 0) for g in sets))
    first = [weigh(g, old, 1.0, ws=ws) for g in sets]
    for _ in range(3):
        for g, (out, new) in zip(sets, first):
            o, n = weigh(g, old, 1.0, ws=ws)
            assert torch.equal(o, out) and torch.equal(n, new)
    outs, news = [torch.zeros_like(o) for o, _ in first], [torch.full_like(n, -7.0) for _, n in first]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for g, o, n in zip(sets, outs, news):
            kl.kl_attention_weights(shape_of(g), g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"],
                                    g["cu_q"], g["q"].shape[0], max(g["news"]), old, 1500, 1.0, n, 0, o, kl.KL_FP32,
                                    ws, err)
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        for o, n, (out, new) in zip(outs, news, first):
            assert torch.equal(o, out) and torch.equal(n, new)
            n.fill_(-7.0)


@pytest.mark.parametrize("n", [2, 6, 40])
def test_a_long_sequence(n):
    x = inputs((40000, 3), (n, 1), 8, 1, 64)
    check(x, 1.0)


@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (64, 1)])
@pytest.mark.parametrize("max_q", [0, 1, 128])
def test_a_call_without_new_tokens(decay, Hq, Hkv, max_q):
    """The weights fade; what was not there stays, and a length that does not fit is reported."""
    x = inputs((300, 5, 0, 1000), (0, 0, 0, 0), Hq, Hkv)
    g = on(x)
    for stride in (1003, 400):
        old = torch.rand(4, Hkv, stride, generator=torch.Generator().manual_seed(2)).cuda()
        for new in (torch.full_like(old, -7.0), old.clone()):
            was, err = new.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
            kl.kl_attention_weights(shape_of(g), None, g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"],
                                    0, max_q, old if decay else None, stride, decay, new, 0, None, kl.KL_BF16, None, err)
            torch.cuda.synchronize()
            assert int(err) == (kl.KL_FLAG_BAD_LENGTH if stride < 1000 else 0)
            for b, L in enumerate((300, 5, 0, 1000)):
                L = L if L <= stride else 0
                assert torch.equal(new[b, :, :L], old[b, :, :L] * decay) and torch.equal(new[b, :, L:], was[b, :, L:])


@pytest.mark.parametrize("Hq,n", [(8, 1), (32, 1), (8, 20)])
def test_more_units_than_shared_counters(Hq, n):
    lens = [n + (7 * b) % 31 for b in range(2100)]
    check(inputs(lens, [n if b % 5 else 0 for b in range(2100)], Hq, 8), 0.5, splits=0 if n == 1 else 3)
