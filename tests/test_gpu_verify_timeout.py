"""Failure detection of the verification operators, without a GPU fault: with the wait limit at one nanosecond the
waits run out on purpose, the call returns and raises KL_FLAG_TIMEOUT, and the next call is right again."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._gpu import to_dev
from tests._verify import tree_inputs, tree_reference
from tests.test_gpu_logprobs import DT, check, make
from tests.test_gpu_timeout import short_waits
from tests.test_gpu_tree import check as check_tree
from tests.test_gpu_tree import run as run_tree

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


@pytest.mark.parametrize("top", [0, 5])
@pytest.mark.parametrize("T,V", [(300, 17000), (700, 60000)])       # (CTAs that wait: several chunks each)
@pytest.mark.parametrize("dtype", DT)
def test_log_probabilities_time_out_then_recover(dtype, T, V, top):
    x, t, _ = make(T, V, dtype, T)
    ws = torch.zeros(max(256, kl.kl_logprobs_workspace_size(T, V, top)), dtype=torch.uint8, device="cuda")
    lp, en, tl = (torch.zeros((T, k), device="cuda") for k in (3, 1, max(top, 1)))
    ti, err = (torch.zeros((n,), dtype=torch.int32, device="cuda") for n in (T * max(top, 1), 1))
    xd, td = x.cuda(), t.to(torch.int32).cuda()
    torch.cuda.synchronize()
    with short_waits(1):
        kl.kl_token_logprobs(T, V, V, xd, DT[dtype], 1.0, td, 3, top, lp, en, tl, ti, ws, err)
        torch.cuda.synchronize()
    assert int(err.item()) & kl.KL_FLAG_TIMEOUT
    ws.zero_()
    check(x, t, top, ws=ws)


@pytest.mark.parametrize("splits", [0, 1])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts, per_q", [((4, 3), False), ((4, 3), True), ((8, 8), False), ((30, 64), False),
                                           ((30, 64), True)])
def test_trees_time_out_then_recover(drafts, per_q, out, splits):
    x = tree_inputs((5000, 3000), drafts, 8, 2, seed=drafts[0], wr_per_query_head=per_q)
    g, T, mq = to_dev(x), x["q"].shape[0], max(drafts)
    sh = kl.make_shape(2, 8, 2, 128, 16, x["v_cache"].shape[0], x["block_table"].shape[1], per_q)
    ws = torch.zeros(max(256, kl.kl_tree_workspace_size(sh, T, mq, splits)), dtype=torch.uint8, device="cuda")
    o = torch.zeros((T, 8, 128), dtype=out, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with short_waits(1):
        kl.kl_tree_attention(sh, g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"],
                             g["parents"], T, mq, splits, o, kl.KL_FP32 if out == torch.float32 else kl.KL_BF16, ws,
                             err)
        torch.cuda.synchronize()
    assert int(err.item()) & kl.KL_FLAG_TIMEOUT
    ws.zero_()
    check_tree(run_tree(x, out, splits=splits, ws=ws), tree_reference(x), out)
