"""kl_window_attention against its definition in 64 bits: windows and first tokens around tiles and pages, head
layouts, lengths, splits, prompts, rows that a position does not see."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import attention, close, inputs, on, shape_of, window, workspace

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def both(x, W, S, **kw):
    g = on(x)
    want = attention(g, W, S, scale=kw.get("scale") or None, composed=kw.get("composed", False))[0]
    for dtype in TYPES:
        close(window(g, W, S, dtype, **kw), want, dtype)


@pytest.mark.parametrize("n", [1, 2])
def test_one_short_sequence(n):
    both(inputs((5,), (n,)), 3, 1)


@pytest.mark.parametrize("W", [1, 2, 63, 64, 65, 127, 128, 129, 300, 5000])
@pytest.mark.parametrize("S", [0, 1, 4, 128, 130, 700])
def test_windows_around_tiles(W, S):
    both(inputs((1, 777, 64, 513, 300), (1, 1, 1, 1, 0)), W, S)
    both(inputs((9, 777, 64, 513, 300), (9, 3, 1, 2, 0)), W, S)


@pytest.mark.parametrize("W", [1, 2, 5, 63, 64, 65, 127, 128, 200, 5000])
@pytest.mark.parametrize("S", [0, 3, 64, 129, 400])
def test_chunks_around_tiles(W, S):
    both(inputs((150, 777, 64, 513, 40), (150, 130, 1, 65, 0), 12, 2), W, S)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (12, 2), (28, 4), (32, 1), (64, 8), (40, 2), (128, 1)])
@pytest.mark.parametrize("per_q", [False, True])
def test_head_layouts(Hq, Hkv, per_q):
    for news in ((1, 1, 0), (4, 1, 2), (17, 33, 1)):
        both(inputs((333, 40, 200), news, Hq, Hkv, seed=Hq, wr_per_query_head=per_q), 100, 5)


@pytest.mark.parametrize("P", [16, 32, 64, 128])
@pytest.mark.parametrize("splits", [0, 1, 2, 3, 7, 64])
def test_pages_and_splits(P, splits):
    for news in ((1, 1, 1), (5, 2, 3), (70, 129, 3)):
        both(inputs((1500, 131, 700), news, 16, 2, P), 900, 70, splits=splits)


@pytest.mark.parametrize("W,S", [(1 << 30, 0), (100, 4), (1000, 64), (1, 0)])
def test_a_prompt(W, S):
    both(inputs((2100,), (2100,), 4, 1), W, S)
    both(inputs((1900, 5, 700), (1900, 5, 700), 6, 3, wr_per_query_head=True), W, S)


def test_scale_and_composed_queries():
    x = inputs((300, 77), (3, 1))
    both(x, 50, 2, scale=0.2)
    both(x, 50, 2, composed=True)
    both(inputs((300, 277), (60, 150)), 50, 2, composed=True)


def test_loose_bound_on_the_rows():
    both(inputs((300, 77), (3, 1)), 50, 2, max_q=40)
    both(inputs((300, 77), (3, 1)), 50, 2, max_q=1000)


@pytest.mark.parametrize("news", [(1, 1), (4, 3), (90, 200)])
@pytest.mark.parametrize("dtype", TYPES)
def test_hidden_pages_are_not_read(news, dtype):
    """Freed pages: other sequences' NaN rows, or ids that no pool has, change nothing and raise nothing."""
    W, S, P = 200, 20, 16
    x = inputs((2000, 1500), news, P=P)
    want = attention(on(x), W, S)[0]
    for b, (L, n) in enumerate(zip((2000, 1500), news)):
        first = (L - n - W + 1) // P
        for i in range(2, first):
            page = int(x["block_table"][b, i])
            x["v_cache"][page] = math.nan if i % 2 else math.inf
            if i % 3 == 0:
                x["block_table"][b, i] = (-1, 1 << 30)[i % 2]
    close(window(on(x), W, S, dtype), want, dtype)


@pytest.mark.parametrize("news", [(1, 1), (4, 3), (90, 200)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, -3e38])
def test_hidden_rows_reach_nothing(news, dtype, bad):
    """Rows in visible pages that no position sees, and the rows behind the sequence."""
    W, S, P, lens = 200, 20, 32, (2000, 1499)
    x = inputs(lens, news, P=P)
    want = attention(on(x), W, S)[0]
    for b, (L, n) in enumerate(zip(lens, news)):
        for t in list(range(S, L - n - W + 1)) + list(range(L, -(-L // P) * P)):
            x["v_cache"][int(x["block_table"][b, t // P]), :, t % P] = bad
    close(window(on(x), W, S, dtype), want, dtype)


@pytest.mark.parametrize("W", [1, 7, 40, 1000])
@pytest.mark.parametrize("n", [3, 30, 150])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_bad_row_reaches_those_who_see_it(W, n, dtype):
    L, S = 500, 3
    for t in (0, L - n - W // 2, L - n, L - n + 1, L - n // 2, L - 1):
        x = inputs((L,), (n,), 8, 2)
        if t < 0:
            continue
        x["v_cache"][int(x["block_table"][0, t // 16]), :, t % 16, 5] = math.nan
        want = attention(on(x), W, S)[0]
        # (bf16 outputs of many rows: a tile's rows of value infinity in fp16 raise the range flag)
        wide = n * 4 <= 32 or dtype == torch.float32
        dirty = bool(torch.isnan(want).any())
        got = window(on(x), W, S, dtype, flags=0 if wide or not dirty else kl.KL_FLAG_RANGE).double()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = ~torch.isnan(want)
        if ok.any():
            close(got[ok], want[ok], dtype)


@pytest.mark.parametrize("news", [(1, 1, 1), (40, 33, 90)])
def test_bad_lengths_and_pages_are_reported(news):
    x = inputs((300, 200, 100), news)
    g = on(x)
    want = attention(g, 64, 4)[0]
    cu = x["cu_q"].tolist()
    for dtype in TYPES:
        for L in (-1, news[1] - 1, 1 << 29):
            g["seq_lens"][1] = L
            got = window(g, 64, 4, dtype, flags=kl.KL_FLAG_BAD_LENGTH)
            g["seq_lens"][1] = 200
            assert torch.isnan(got[cu[1]:cu[2]].float()).all()
            for a, b in ((0, cu[1]), (cu[2], cu[3])):
                close(got[a:b], want[a:b], dtype)
        old = int(g["block_table"][1, 11])
        for page in (-1, x["num_pages"]):
            g["block_table"][1, 11] = page
            # (the outputs of those who see the page are unspecified, and where they are not finite, in range or not)
            got = window(g, 64, 4, dtype, flags=kl.KL_FLAG_BAD_PAGE, maybe=kl.KL_FLAG_RANGE)
            close(got[:cu[1]], want[:cu[1]], dtype)
        g["block_table"][1, 11] = old


def test_more_rows_than_announced_are_refused_on_the_device():
    g = on(inputs((300, 200), (5, 4)))
    got = window(g, 64, 4, max_q=4, flags=kl.KL_FLAG_BAD_LENGTH)
    assert torch.isnan(got[:5]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_a_shared_workspace_and_a_graph(dtype):
    """Calls of several forms over one workspace, eager and replayed with other lengths."""
    W, S = 300, 5
    sets = [on(inputs((1500, 40, 800), n, 16, 2, seed=i)) for i, n in enumerate(((1, 1, 1), (3, 2, 4), (100, 1, 300)))]
    sizes = [kl.kl_window_workspace_size(shape_of(g), g["q"].shape[0], max(g["news"]), W, S, 0) for g in sets]
    ws = workspace(max(sizes))
    for _ in range(2):
        for g in sets:
            close(window(g, W, S, dtype, ws=ws), attention(g, W, S)[0], dtype)
    outs = [torch.empty(g["q"].shape, dtype=dtype, device="cuda") for g in sets]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def calls():
        for g, out in zip(sets, outs):
            kl.kl_window_attention(shape_of(g), g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"],
                                   g["cu_q"], g["q"].shape[0], max(g["news"]), W, S, 0, out,
                                   kl.KL_FP32 if dtype == torch.float32 else kl.KL_BF16, ws, err)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for lens in ((1500, 40, 800), (1100, 33, 500), (700, 1, 301)):
        for g, out in zip(sets, outs):
            g["seq_lens"].copy_(torch.tensor([max(L, n) for L, n in zip(lens, g["news"])]))
            out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        assert int(err) == 0
        for g, out in zip(sets, outs):
            close(out, attention(g, W, S)[0], dtype)


def test_results_are_the_same_on_every_run():
    for news in ((1, 1, 1), (3, 2, 4), (100, 1, 300)):
        g = on(inputs((1500, 40, 800), news, 16, 2))
        for dtype in TYPES:
            a = window(g, 300, 5, dtype)
            for _ in range(5):
                assert torch.equal(window(g, 300, 5, dtype), a)


@pytest.mark.parametrize("L", [4096, 4097, 4200, 8192, 8300, 20000])
@pytest.mark.parametrize("grow", [0.0, 3.0])
def test_long_lines(L, grow):
    """Many tiles per block, with scores that stay alike or grow along the sequence (the references move)."""
    x = inputs((L, 300), (40, 40), 4, 1, 64)
    if grow:
        up = torch.linspace(0.2, grow, L)
        for t in range(L):
            x["v_cache"][int(x["block_table"][0, t // 64]), :, t % 64] *= up[t].to(torch.bfloat16)
    for W in (1 << 30, L - 100):
        both(x, W, 3)


@pytest.mark.parametrize("n", [1, 200])
def test_another_stream(n):
    g = on(inputs((900,), (n,), 16, 2))
    want = attention(g, 100, 4)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = window(g, 100, 4)
    close(got, want)


def test_a_long_cache_beyond_32_bits():
    """A pool of more than 2^31 values, the last pages of which a sequence reads."""
    pages, Hkv, P = 140000, 8, 16
    v = torch.empty(pages, Hkv, P, 128, dtype=torch.bfloat16, device="cuda")
    x = inputs((700, 300), (1, 1), 16, 8, P)
    g = on(x)
    used = g["v_cache"].shape[0]
    v[pages - used:] = g["v_cache"]
    g["block_table"] = torch.where(g["block_table"] >= 0, g["block_table"] + (pages - used), -1).to(torch.int32)
    want = attention(on(x), 400, 4)[0]
    g["v_cache"] = v
    for dtype in TYPES:
        close(window(g, 400, 4, dtype), want, dtype)
    x = inputs((700, 300), (70, 100), 16, 8, P)
    want = attention(on(x), 400, 4)[0]
    g2 = on(x)
    v[pages - used:] = g2["v_cache"]
    g2["block_table"] = torch.where(g2["block_table"] >= 0, g2["block_table"] + (pages - used), -1).to(torch.int32)
    g2["v_cache"] = v
    for dtype in TYPES:
        close(window(g2, 400, 4, dtype), want, dtype)


@pytest.mark.parametrize("Hq,n", [(8, 1), (32, 1), (8, 20), (32, 40)])
@pytest.mark.parametrize("splits", [0, 3])
def test_more_units_than_shared_counters(Hq, n, splits):
    lens = [n + (7 * b) % 331 for b in range(2100)]
    both(inputs(lens, [n if b % 5 else 0 for b in range(2100)], Hq, 8), 150, 3, splits=splits)
