"""kl_tree_attention against its definition in 64 bits: tree shapes, head layouts, lengths around tiles and
pages, splits, both forms of W^R and the composed query, values in rows that a draft does not see."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests import _gpu
from tests._gpu import ATOL, RTOL, to_dev
from tests._verify import REL, tree_inputs, tree_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def run(x, out_dtype=torch.float32, splits=0, scale=0.0, composed=False, max_q=None, ws=None, flags=0):
    g = to_dev(x)
    T, Hq, D = x["q"].shape
    pages, Hkv, P, _ = x["v_cache"].shape
    sh = kl.make_shape(len(x["drafts"]), Hq, Hkv, D, P, pages, x["block_table"].shape[1],
                       x["wr_per_query_head"], scale)
    max_q = max_q or max(1, max(x["drafts"]))
    out = torch.full((T, Hq, D), float("nan"), dtype=out_dtype, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    need = kl.kl_tree_workspace_size(sh, T, max_q, splits)
    ws = torch.zeros(max(256, need), dtype=torch.uint8, device="cuda") if ws is None else ws
    kl.kl_tree_attention(sh, g["q"], None if composed else g["w_r"], g["v_cache"], g["block_table"],
                         g["seq_lens"], g["cu_q"], g["parents"], T, max_q, splits, out,
                         kl.KL_FP32 if out_dtype == torch.float32 else kl.KL_BF16, ws, err)
    torch.cuda.synchronize()
    assert int(err.item()) == flags
    if need:                                       # counters are back at zero
        assert not ws[:65536].any()
    return out.cpu()


def check(got, want, dtype=None):
    dtype = dtype or got.dtype
    assert torch.isfinite(got.float()).all()
    d = got.double() - want
    assert float(d.norm()) <= REL[dtype] * float(want.norm()) + 1e-12
    assert bool((d.abs() <= ATOL + RTOL * want.abs()).all())


@pytest.mark.parametrize("kind", ["chain", "star", "binary", "random"])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_tree_shapes(kind, out):
    x = tree_inputs((300, 61, 129, 17), (12, 61, 33, 1), kind=kind)
    check(run(x, out), tree_reference(x), out)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (12, 2), (28, 4), (32, 1), (64, 8), (71, 1), (128, 1)])
@pytest.mark.parametrize("per_q", [False, True])
def test_head_layouts(Hq, Hkv, per_q):
    x = tree_inputs((200, 40), (9, 16), Hq, Hkv, wr_per_query_head=per_q, seed=Hq)
    want = tree_reference(x)
    check(run(x), want)
    check(run(x, torch.bfloat16), want, torch.bfloat16)


@pytest.mark.parametrize("n", [1, 2, 21, 22, 32, 33, 63, 64, 65, 127, 128])
@pytest.mark.parametrize("committed", [0, 1, 63, 64, 65, 127, 128, 200, 1000])
def test_lengths_around_tiles(n, committed):
    x = tree_inputs((committed + n, committed + 1), (n, 1), 6, 1, seed=n + committed)
    want = tree_reference(x)
    check(run(x), want)
    check(run(x, torch.bfloat16), want, torch.bfloat16)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
def test_pages_and_splits(P, splits):
    x = tree_inputs((1500, 3, 131, 700, 129), (20, 3, 5, 0, 1), 8, 2, P=P, seed=P)
    check(run(x, splits=splits), tree_reference(x))


# Few rows per value head (drafts x heads of a group up to 32) with bf16 outputs: CTAs of 16 and of 32 rows, one
# and two to an SM.
@pytest.mark.parametrize("Hq,Hkv,n", [(1, 1, 1), (1, 1, 17), (1, 1, 32), (4, 1, 4), (8, 2, 8), (6, 1, 5), (16, 1, 2),
                                      (32, 1, 1), (5, 1, 3), (40, 8, 6)])
@pytest.mark.parametrize("committed", [0, 1, 127, 128, 300])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_few_rows(Hq, Hkv, n, committed, splits):
    x = tree_inputs((committed + n, committed + max(1, n // 2), 900, 0), (n, max(1, n // 2), min(n, 2), 0), Hq, Hkv,
                    seed=n + committed)
    check(run(x, torch.bfloat16, splits=splits), tree_reference(x), torch.bfloat16)


@pytest.mark.parametrize("n", [2, 4, 8])
def test_few_rows_of_many_sequences(n):
    lens = tuple(60 + 37 * (i % 11) for i in range(90))
    x = tree_inputs(lens, tuple(1 + i % n for i in range(90)), 8, 2, seed=n)
    check(run(x, torch.bfloat16), tree_reference(x), torch.bfloat16)
    check(run(x, torch.bfloat16, composed=True), tree_reference(x, composed=True), torch.bfloat16)


def test_few_rows_of_a_long_cache():
    x = tree_inputs((30000, 5000), (8, 3), 8, 2, P=32, seed=78)
    want = tree_reference(x)
    for splits in (0, 1, 40):
        check(run(x, torch.bfloat16, splits=splits), want, torch.bfloat16)


@pytest.mark.parametrize("splits", [0, 4])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_few_rows_and_a_row_that_is_not_finite(value, splits):
    x = tree_inputs((530, 140), (8, 7), 8, 2, seed=11)
    want = tree_reference(x)
    P, cu, bad = 16, x["cu_q"].tolist(), {0: 2, 1: 0}
    for b, i in bad.items():
        t = int(x["seq_lens"][b]) - x["drafts"][b] + i
        x["v_cache"][int(x["block_table"][b, t // P]), :, t % P, 5] = value
        L = int(x["seq_lens"][b])
        x["v_cache"][int(x["block_table"][b, L // P]), :, L % P:] = math.nan      # behind the end
    got = run(x, torch.bfloat16, splits=splits)
    for b in range(2):
        for i in range(x["drafts"][b]):
            j = i
            while j > bad[b]:
                j = int(x["parents"][cu[b] + j])
            r = cu[b] + i
            if j != bad[b]:
                d = got[r].double() - want[r]
                assert float(d.norm() / want[r].norm()) < 4 * REL[torch.bfloat16], (b, i)
            elif math.isnan(value):
                assert torch.isnan(got[r].float()).all(), (b, i)


def test_few_rows_flags():
    x = tree_inputs((100, 50, 80), (5, 5, 8))
    want = tree_reference(x)
    y = dict(x, parents=x["parents"].clone())
    y["parents"][7] = 2                           # sequence 1, draft 2: itself
    got = run(y, torch.bfloat16, flags=kl.KL_FLAG_BAD_TREE)
    check(got[:5], want[:5])
    y = dict(x, seq_lens=x["seq_lens"].clone())
    y["seq_lens"][1] = 4                          # fewer rows than drafts
    got = run(y, torch.bfloat16, flags=kl.KL_FLAG_BAD_LENGTH)
    check(got[10:], want[10:])
    assert torch.isnan(got[5:10].float()).all()


def test_no_drafts_anywhere_but_one():
    x = tree_inputs((100, 50, 80), (0, 0, 7))
    check(run(x), tree_reference(x))


def test_single_tokens_are_the_decode():
    x = tree_inputs((700, 1, 300, 64), (1, 1, 1, 1), 32, 8)
    got = run(x)
    y = dict(x, workload=None)
    sh = kl.make_shape(4, 32, 8, 128, 16, x["v_cache"].shape[0], x["block_table"].shape[1])
    out, err = _gpu.decode(to_dev(y), sh)
    assert err == 0
    assert float((got - out.cpu()).norm() / out.cpu().norm()) < 2 * REL[torch.float32]


def test_composed_query_and_scale():
    x = tree_inputs((500, 260), (40, 7), 12, 2)
    check(run(x, composed=True), tree_reference(x, composed=True))
    check(run(x, scale=0.25), tree_reference(x, scale=0.25))


def test_a_larger_bound_and_a_shared_workspace():
    x = tree_inputs((1500, 260), (40, 7), 12, 2)
    ws = torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")
    want = tree_reference(x)
    for max_q, splits in ((128, 5), (40, 0), (64, 3)):
        check(run(x, max_q=max_q, splits=splits, ws=ws), want)


def test_bf16_outputs_of_large_scores():
    """One fp16 operand each for query and weights (more than 32 rows) or bf16 pairs (fewer): against scores of tens
    of units, whose weights the fp16 query moves by up to |s| 2^-12."""
    for drafts in ((30, 64), (8, 5)):
        x = tree_inputs((900, 333), drafts, 8, 2)
        x["q"] = (x["q"].float() * 6).to(torch.bfloat16)
        want = tree_reference(x)
        d = run(x, torch.bfloat16).double() - want
        assert float(d.norm() / want.norm()) < (60 * 2.0 ** -12 if drafts[0] > 8 else REL[torch.bfloat16])


def test_large_scores_and_outliers():
    x = tree_inputs((900, 333), (30, 64), 8, 2)
    x["q"] = (x["q"].float() * 6).to(torch.bfloat16)
    gen = torch.Generator().manual_seed(1)
    v = x["v_cache"]
    x["v_cache"] = torch.where(torch.rand(v.shape, generator=gen) < 0.01, v * 20, v)
    want = tree_reference(x)
    d = run(x).double() - want
    # scores of up to a few hundred: errors of 2^-17 of that in the exponent
    assert float(d.norm() / want.norm()) < 2e-3
    assert bool((d.abs() <= ATOL + RTOL * want.abs() * 2).all())


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_a_row_that_is_not_finite_reaches_those_who_see_it(value):
    x = tree_inputs((150, 90), (40, 70), 8, 2, kind="random", seed=9)
    want = tree_reference(x)
    P, cu = 16, x["cu_q"].tolist()
    bad = {0: 5, 1: 33}
    for b, i in bad.items():
        t = int(x["seq_lens"][b]) - x["drafts"][b] + i
        x["v_cache"][int(x["block_table"][b, t // P]), :, t % P, ::7] = value
    got = run(x)
    for b in range(2):
        for i in range(x["drafts"][b]):
            j = i
            while j > bad[b]:
                j = int(x["parents"][cu[b] + j])
            r = cu[b] + i
            if j != bad[b]:
                d = got[r].double() - want[r]
                assert float(d.norm() / want[r].norm()) < 4 * REL[torch.float32], (b, i)
            elif math.isnan(value):
                assert torch.isnan(got[r]).all(), (b, i)


def test_half_precision_outputs_and_values_beyond_it():
    """bf16 outputs take the values in fp16: a drafted row beyond its range, or not finite, reaches those who
    see it alone; a committed one raises the flag."""
    x = tree_inputs((150, 90), (40, 70), 8, 2, kind="random", seed=9)
    cu = x["cu_q"].tolist()
    P = 16
    x["v_cache"][0, 0, 0, 0] = 65280.0
    want = tree_reference(x)
    y = dict(x, v_cache=x["v_cache"].clone())
    bad = {0: 5, 1: 33}
    for (b, i), value in zip(bad.items(), (70000.0, math.inf)):
        t = int(x["seq_lens"][b]) - x["drafts"][b] + i
        y["v_cache"][int(x["block_table"][b, t // P]), :, t % P, 3::40] = value
    got = run(y, torch.bfloat16, flags=kl.KL_FLAG_RANGE)
    for b in range(2):
        for i in range(x["drafts"][b]):
            j = i
            while j > bad[b]:
                j = int(x["parents"][cu[b] + j])
            r = cu[b] + i
            if j != bad[b]:
                d = got[r].double() - want[r]
                assert float(d.norm() / want[r].norm()) < 4 * REL[torch.bfloat16], (b, i)
            else:
                assert torch.isnan(got[r].float()).all(), (b, i)
    y = dict(x, v_cache=x["v_cache"].clone())
    y["v_cache"][int(x["block_table"][0, 0]), :, 3, 5] = 70000.0
    run(y, torch.bfloat16, flags=kl.KL_FLAG_RANGE)
    check(run(y)[cu[1]:], tree_reference(y)[cu[1]:])


def test_rows_past_the_end_and_unused_pages_may_hold_anything():
    x = tree_inputs((150, 33), (17, 33), 8, 2)
    want = tree_reference(x)
    for b in range(2):
        L = int(x["seq_lens"][b])
        if L % 16:
            x["v_cache"][int(x["block_table"][b, L // 16]), :, L % 16:] = math.nan
    check(run(x), want)


def test_page_permutation_is_bit_exact():
    x = tree_inputs((1000, 500), (30, 12), 8, 2, table="identity")
    a = run(x, splits=3)
    perm = torch.randperm(x["v_cache"].shape[0], generator=torch.Generator().manual_seed(3))
    y = dict(x, v_cache=torch.empty_like(x["v_cache"]))
    y["v_cache"][perm] = x["v_cache"]
    bt = x["block_table"].clone()
    y["block_table"] = torch.where(bt >= 0, perm[bt.long().clamp_min(0)].to(torch.int32), bt)
    assert torch.equal(a, run(y, splits=3))
    assert torch.equal(a, run(x, splits=3))


def test_flags():
    x = tree_inputs((100, 50, 80), (10, 5, 8))
    want = tree_reference(x)
    y = dict(x, parents=x["parents"].clone())
    y["parents"][12] = 2                          # sequence 1, draft 2: itself
    got = run(y, flags=kl.KL_FLAG_BAD_TREE)
    check(got[:10], want[:10])
    y = dict(x, seq_lens=x["seq_lens"].clone())
    y["seq_lens"][1] = 4                          # fewer rows than drafts
    got = run(y, flags=kl.KL_FLAG_BAD_LENGTH)
    check(got[15:], want[15:])
    assert torch.isnan(got[10:15]).all()
    y = dict(x, block_table=x["block_table"].clone())
    y["block_table"][1, 0] = x["v_cache"].shape[0]
    got = run(y, flags=kl.KL_FLAG_BAD_PAGE)
    check(torch.cat([got[:10], got[15:]]), torch.cat([want[:10], want[15:]]))


def test_a_missing_or_small_workspace_is_refused():
    x = tree_inputs((300,), (5,))
    for ws in (torch.zeros(1000, dtype=torch.uint8, device="cuda"), torch.zeros(1 << 23, dtype=torch.uint8, device="cuda")[8:]):
        with pytest.raises(kl.KLError) as e:
            run(x, ws=ws)
        assert e.value.status == kl.KL_ERR_WORKSPACE


def test_another_stream_and_a_graph():
    x = tree_inputs((1200, 300), (20, 33), 8, 2)
    g, want = to_dev(x), tree_reference(x)
    T = x["q"].shape[0]
    sh = kl.make_shape(2, 8, 2, 128, 16, x["v_cache"].shape[0], x["block_table"].shape[1])
    ws = torch.zeros(max(256, kl.kl_tree_workspace_size(sh, T, 33, 4)), dtype=torch.uint8, device="cuda")
    out = torch.zeros((T, 8, 128), device="cuda")
    q = torch.zeros_like(g["q"])

    def call():
        kl.kl_tree_attention(sh, q, g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"],
                             g["parents"], T, 33, 4, out, kl.KL_FP32, ws)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        q.copy_(g["q"])
        call()
    side.synchronize()
    check(out.cpu(), want)
    graph = torch.cuda.CUDAGraph()
    q.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        q.copy_(g["q"])
        call()
    out.zero_()
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    check(out.cpu(), want)


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,drafts", [
    ((20000, 3, 700, 1, 5000), (5, 3, 64, 1, 33)),       # runs that end inside units of one long sequence
    ((500,) * 90, (7,) * 90),                             # more units than CTAs
    ((260, 17, 0, 128, 129, 384) * 70, (1, 2, 0, 3, 4, 5) * 70)])   # more sequences than threads
def test_runs_of_many_lengths(lens, drafts, out):
    x = tree_inputs(lens, drafts, 8, 2, seed=len(lens))
    want = tree_reference(x)
    for splits in (0, 1, 3):
        check(run(x, out, splits=splits), want, out)


def test_a_long_cache():
    x = tree_inputs((40000,), (24,), 8, 1, P=64, seed=77)
    for splits in (0, 1):
        check(run(x, splits=splits), tree_reference(x))
    check(run(x, torch.bfloat16), tree_reference(x), torch.bfloat16)
    assert np.isfinite(run(x).numpy()).all()


@pytest.mark.parametrize("splits", [1, 2])
def test_fp32_sums_of_a_long_cache_with_outliers(splits):
    # A few tokens of large scores hold most of the weight, so that each of the others is small against the sum.
    # Scores reach about 32 in units of log2: a score product adds eight K steps, each of which truncates on
    # average half of 2^-19 there, so a weight may be off by 8 x 2^-20 x ln 2; the sums add their own few 2^-24.
    x = tree_inputs((64615,), (2,), Hq=4, Hkv=4, P=32, kind="chain", seed=9)
    v = x["v_cache"]
    big = torch.rand(v.shape, generator=torch.Generator().manual_seed(77)) < 0.01
    x["v_cache"] = torch.where(big, v / v.float().std() * 20, v / v.float().std()).to(torch.bfloat16)
    want = tree_reference(x, composed=True)
    d = run(x, torch.float32, splits=splits, composed=True).double() - want
    assert float(d.norm()) <= (8 * 2.0 ** -20 * math.log(2) + 2.0 ** -22) * float(want.norm())


@pytest.mark.parametrize("Hq,Hkv,n", [(1, 1, 7), (4, 1, 4), (8, 2, 8), (6, 1, 5), (16, 1, 2), (20, 1, 1), (32, 1, 1),
                                      (11, 1, 2), (40, 8, 6), (15, 3, 3)])
@pytest.mark.parametrize("per_q", [False, True])
@pytest.mark.parametrize("splits", [0, 3])
def test_few_rows_of_either_type(Hq, Hkv, n, per_q, splits):
    # blocks of 16 rows that hold a part of a group's heads, or the same head of several drafts
    x = tree_inputs((500 + n, n, 131, 1), (n, max(1, n // 2), min(n, 2), 0), Hq, Hkv, wr_per_query_head=per_q,
                    seed=Hq + n)
    want = tree_reference(x)
    check(run(x, splits=splits), want)
    check(run(x, torch.bfloat16, splits=splits), want, torch.bfloat16)


def test_few_rows_of_many_sequences_and_w_r_per_query_head():
    lens = tuple(60 + 37 * (i % 11) for i in range(90))
    x = tree_inputs(lens, tuple(1 + i % 4 for i in range(90)), 8, 2, wr_per_query_head=True, seed=4)
    want = tree_reference(x)
    check(run(x), want)
    check(run(x, torch.bfloat16), want, torch.bfloat16)
