"""kl_tree_attention in blocks of 128 rows (more than 32 rows per value head): bf16 outputs with composed queries, scales,
page sizes and in a captured graph; the error of fp32 outputs on a long cache with outliers."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._gpu import to_dev
from tests._verify import tree_inputs, tree_reference
from tests.test_gpu_tree import check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_bf16_pages_and_queries(P, splits):
    x = tree_inputs((1500, 260, 128, 129), (40, 7, 0, 64), 12, 2, P=P, seed=P)
    check(run(x, torch.bfloat16, splits=splits), tree_reference(x))
    check(run(x, torch.bfloat16, splits=splits, composed=True), tree_reference(x, composed=True))
    check(run(x, torch.bfloat16, splits=splits, scale=0.25), tree_reference(x, scale=0.25))


def test_bf16_more_segments_than_ctas():
    # every CTA goes through several sequences, whose blocks fill one to four quarters of the 128 rows
    lens = tuple(130 + 71 * (i % 13) for i in range(120))
    x = tree_inputs(lens, tuple(1 + 7 * i % 33 for i in range(120)), 8, 2, seed=8)
    want = tree_reference(x)
    for splits in (0, 1):
        check(run(x, torch.bfloat16, splits=splits), want)
    check(run(x), want, torch.float32)


def test_bf16_in_a_graph():
    x = tree_inputs((1200, 300), (20, 33), 8, 2)
    g, want, T = to_dev(x), tree_reference(x), x["q"].shape[0]
    sh = kl.make_shape(2, 8, 2, 128, 16, x["v_cache"].shape[0], x["block_table"].shape[1])
    ws = torch.zeros(max(256, kl.kl_tree_workspace_size(sh, T, 33, 4)), dtype=torch.uint8, device="cuda")
    out = torch.zeros((T, 8, 128), dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kl.kl_tree_attention(sh, g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"],
                             g["parents"], T, 33, 4, out, kl.KL_BF16, ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(out.cpu(), want)


@pytest.mark.parametrize("splits", [0, 1, 2, 7])
def test_fp32_sums_with_outliers(splits):
    # A few tokens of large scores hold most of the weight. Scores reach about 32 in units of log2: the eight steps of
    # their leading product truncate up to a unit of 2^-19 each, at rms sqrt(8 / 12) of one against their mean, which
    # all tokens share. A token's weight is off by ln 2 of that, the outputs by no more; the bound is twice the rms.
    # (Query and weights in two bf16 terms: 2^-18 of the score, several times that.)
    x = tree_inputs((64615,), (40,), Hq=1, Hkv=1, P=32, kind="chain", seed=9)
    v = x["v_cache"]
    big = torch.rand(v.shape, generator=torch.Generator().manual_seed(77)) < 0.01
    x["v_cache"] = torch.where(big, v / v.float().std() * 20, v / v.float().std()).to(torch.bfloat16)
    want = tree_reference(x, composed=True)
    d = run(x, torch.float32, splits=splits, composed=True).double() - want
    assert float(d.norm()) <= 2 * 2.0 ** -19 * math.sqrt(8 / 12) * math.log(2) * float(want.norm())
