"""kl_evict against its definition: what stays, its order, ties, moves in place and to other pages, refusals."""
from __future__ import annotations

import math
import random

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import keep, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def case(lens, Hkv=2, D=128, P=16, kind="random", seed=7, spare=0, stride=None):
    """A cache of tagged rows, its table, and weights of a kind."""
    gen = torch.Generator().manual_seed(seed)
    B, pages = len(lens), [-(-L // P) for L in lens]
    extra = sum(pages) if spare else 0
    perm = torch.randperm(sum(pages) + extra, generator=gen).to(torch.int32)
    table = torch.full((B, max(1, max(pages))), -1, dtype=torch.int32)
    other = table.clone()
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        if spare:
            other[b, :n] = perm[sum(pages) + at:sum(pages) + at + n]
        at += n
    v = torch.randint(-32768, 32767, (sum(pages) + extra, Hkv, P, D), generator=gen).to(torch.int16)
    E = stride or max(1, max(lens))
    if kind == "random":
        w = torch.rand(B, Hkv, E, generator=gen)
    elif kind == "skewed":
        w = (-torch.log(torch.rand(B, Hkv, E, generator=gen).clamp_min(1e-7))) ** 4 * 1e-3
    elif kind == "ties":
        w = torch.randint(0, 3, (B, Hkv, E), generator=gen).float()
    elif kind == "zero":
        w = torch.zeros(B, Hkv, E)
    elif kind == "rising":
        w = torch.arange(E).float().expand(B, Hkv, E).clone()
    elif kind == "falling":
        w = -torch.arange(E).float().expand(B, Hkv, E) + E
    elif kind == "odd":
        w = torch.rand(B, Hkv, E, generator=gen)
        pick = torch.randint(0, 8, w.shape, generator=gen)
        for i, x in enumerate((math.inf, math.nan, -1.0, -math.inf, 1e-42, 3e38)):
            w[pick == i] = x
    return dict(v=v, table=table, other=other if spare else table, w=w.contiguous(), lens=list(lens), P=P)


def reference(c, budget, sinks, recent):
    """(kept, new_lens, new weights with None where nothing is written, rows per (b, g))."""
    out = []
    for b, L in enumerate(c["lens"]):
        for g in range(c["v"].shape[1]):
            ids = keep(c["w"][b, g].tolist(), L, budget, sinks, recent)
            rows = torch.stack([c["v"][int(c["table"][b, t // c["P"]]), g, t % c["P"]] for t in ids]) if ids else None
            out.append((b, g, L, ids, rows))
    return out


def run(c, budget, sinks, recent, in_place=False, ws=None, flags=0, clones=True):
    B, Hkv, E = c["w"].shape
    num_pages, _, P, D = c["v"].shape
    sh = kl.make_shape(B, Hkv, Hkv, D, P, num_pages, c["table"].shape[1])
    g = {k: c[k].cuda() for k in ("v", "table", "other", "w")}
    if c["other"] is c["table"]:
        g["other"] = g["table"]
    lens = torch.tensor(c["lens"], dtype=torch.int32).cuda()
    new = g["w"] if in_place else torch.full((B, Hkv, E), -7.0, device="cuda")
    new_lens = lens if in_place else torch.full_like(lens, -7)
    kept = torch.full((B, Hkv, budget), -7, dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    need = kl.kl_evict_workspace_size(sh, E, budget)
    ws = workspace(need) if ws is None else ws
    kl.kl_evict(sh, g["w"], E, budget, sinks, recent, g["table"], lens, g["other"], g["v"], new, kept, new_lens, ws, err)
    torch.cuda.synchronize()
    assert int(err) == flags
    assert not ws[:65536].any()
    return kept.cpu(), new_lens.cpu(), new.cpu(), g["v"].cpu()


def check(c, budget, sinks, recent, in_place=False, **kw):
    kept, new_lens, new, v = run(c, budget, sinks, recent, in_place, **kw)
    changed = torch.zeros(v.shape[:3], dtype=torch.bool)
    for b, g, L, ids, rows in reference(c, budget, sinks, recent):
        m = len(ids)
        assert int(new_lens[b]) == m
        assert kept[b, g, :m].tolist() == ids and (kept[b, g, m:] == -1).all()
        want = c["w"][b, g, ids]
        assert torch.equal(new[b, g, :m].view(torch.int32), want.view(torch.int32))
        assert (new[b, g, m:L] == 0).all()
        rest = new[b, g, L:]
        assert torch.equal(rest.view(torch.int32), c["w"][b, g, L:].view(torch.int32)) if in_place else (rest == -7).all()
        for j in range(m):
            page, r = int(c["other"][b, j // c["P"]]), j % c["P"]
            changed[page, g, r] = True
        if m:
            j = torch.arange(m)
            got = v[c["other"][b, j // c["P"]].long(), g, j % c["P"]]
            assert torch.equal(got, rows)
    assert torch.equal(v[~changed], c["v"][~changed])


KINDS = ["random", "skewed", "ties", "zero", "rising", "falling", "odd"]


@pytest.mark.parametrize("sinks,recent,budget", [(6000, 0, 9000), (6000, 9000, 16000), (2560, 1, 2562), (19000, 900, 19901),
                                                 (0, 18000, 18100)])
def test_first_and_last_tokens_beyond_a_piece(sinks, recent, budget):
    """A cluster's CTAs whose piece of the weights lies wholly among the first or the last tokens count none of it."""
    for kind in ("random", "rising"):
        check(case((20000,), Hkv=1, kind=kind), budget, sinks, recent)
        check(case((20000, 6001), Hkv=1, D=64, kind=kind, spare=1), budget, sinks, recent)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("spare", [0, 1])
def test_kinds_of_weights(kind, spare):
    c = case((500, 1, 300, 0, 64, 129), kind=kind, spare=spare)
    for budget, sinks, recent in ((64, 4, 16), (1, 0, 0), (300, 0, 0), (20, 20, 0), (20, 0, 20), (20, 7, 13), (600, 1, 1)):
        check(c, budget, sinks, recent)
        check(c, budget, sinks, recent, in_place=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [1, 8, 16, 32, 100, 128])
@pytest.mark.parametrize("Hkv", [1, 3, 8])
def test_layouts(D, P, Hkv):
    for spare in (0, 1):
        check(case((700, 333, 10), Hkv, D, P, spare=spare), 100, 3, 5)


@pytest.mark.parametrize("L", [2047, 2048, 2049, 5000, 9001, 20000])
@pytest.mark.parametrize("kind", ["skewed", "ties", "odd"])
def test_long_sequences(L, kind):
    for spare in (0, 1):
        check(case((L, L // 2), 1, 64, 16, kind=kind, spare=spare, stride=L + 3), L // 3, 4, 100)


@pytest.mark.parametrize("kind", ["skewed", "zero"])
def test_the_longest(kind):
    L = kl.KL_EVICT_MAX_TOKENS
    check(case((L,), 1, 64, 128, kind=kind, stride=L), 3001, 4, 100)


def test_many_units():
    check(case([random.Random(3).randint(0, 400) for _ in range(70)], 8, 64, 16), 150, 4, 20)


@pytest.mark.parametrize("B", [5, 6, 12, 40])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spare", [0, 1])
def test_numbers_of_units(B, D, spare):
    """40 to 480 value heads in all: each form of the move, with several turns of its CTAs."""
    r = random.Random(B)
    lens = [r.randint(1, 1400) for _ in range(B)]
    check(case(lens, 8, D, 16, spare=spare, kind="skewed"), 800, 4, 100)


@pytest.mark.parametrize("budget", [2999, 2900, 1500, 70])
@pytest.mark.parametrize("kind", ["rising", "falling", "random"])
def test_one_long_unit_in_place(budget, kind):
    """Rows that move by one place, by all that was evicted at once, or by more and more."""
    check(case((3000,), 1, 128, 16, kind=kind), budget, 2, 5)
    check(case((60000,), 1, 64, 16, kind=kind), 20 * budget, 2, 5)


def test_a_budget_of_one_less():
    for kind in ("rising", "falling", "random"):
        c = case((4000, 3999, 4001), 2, 128, 16, kind=kind)
        for budget in (3999, 4000, 1):
            check(c, budget, 0, 0)


def test_some_pages_stay_and_others_are_new():
    c = case((640, 300), spare=1)
    c["other"][:, :10] = c["table"][:, :10]
    check(c, 400, 4, 16)


def test_bad_lengths_and_pages_leave_the_sequence():
    for field, value, flag in (("lens", -1, kl.KL_FLAG_BAD_LENGTH), ("lens", 1 << 20, kl.KL_FLAG_BAD_LENGTH),
                               ("lens", 501, kl.KL_FLAG_BAD_LENGTH), ("table", -1, kl.KL_FLAG_BAD_PAGE),
                               ("table", 1 << 20, kl.KL_FLAG_BAD_PAGE), ("other", -1, kl.KL_FLAG_BAD_PAGE),
                               ("other", 1 << 20, kl.KL_FLAG_BAD_PAGE)):
        c = case((500, 300, 128), spare=1)
        whole = dict(c, table=c["table"].clone(), lens=list(c["lens"]))
        if field == "lens":
            c["lens"][1] = value
        else:
            c[field][1, {"table": 18, "other": 2}[field]] = value
        kept, new_lens, new, v = run(c, 64, 4, 16, flags=flag)
        assert (kept[1] == -7).all() and int(new_lens[1]) == -7 and (new[1] == -7).all()
        for b, g, L, ids, rows in reference(whole, 64, 4, 16):
            if b == 1:
                continue
            assert kept[b, g].tolist() == ids and int(new_lens[b]) == 64
            j = torch.arange(64)
            assert torch.equal(v[c["other"][b, j // 16].long(), g, j % 16], rows)


def test_a_graph_evicts_again_and_again():
    """Captured once, replayed while the weights change: the same as eager calls."""
    c = case((900, 500), 2, 64)
    B, Hkv, E = c["w"].shape
    sh = kl.make_shape(B, Hkv, Hkv, 64, 16, c["v"].shape[0], c["table"].shape[1])
    g = {k: c[k].cuda() for k in ("v", "table", "w")}
    lens = torch.tensor(c["lens"], dtype=torch.int32).cuda()
    kept = torch.zeros(B, Hkv, 300, dtype=torch.int32, device="cuda")
    ws = workspace(kl.kl_evict_workspace_size(sh, E, 300))

    def call():
        kl.kl_evict(sh, g["w"], E, 300, 4, 16, g["table"], lens, g["table"], g["v"], g["w"], kept, lens, ws)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    state = [t.clone() for t in (g["v"], g["w"], lens)]
    for _ in range(3):
        graph.replay()
        lens += 50
        g["w"] += torch.arange(E, device="cuda").remainder(7)
    torch.cuda.synchronize()
    got = [t.clone() for t in (g["v"], g["w"], lens, kept)]
    for t, s in zip((g["v"], g["w"], lens), state):
        t.copy_(s)
    for _ in range(3):
        call()
        lens += 50
        g["w"] += torch.arange(E, device="cuda").remainder(7)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, (g["v"], g["w"], lens, kept)))


@pytest.mark.parametrize("spare", [0, 1])
def test_many_sequences(spare):
    check(case([1 + (7 * b) % 41 for b in range(2100)], Hkv=8, D=64, kind="ties", spare=spare), 19, 2, 5)
