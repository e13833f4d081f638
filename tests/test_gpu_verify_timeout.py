"""Failure detection of the verification operators, without a GPU fault: with the wait limit at one nanosecond the
waits run out on purpose, the call returns and raises KL_FLAG_TIMEOUT, and the next call is right again."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests.test_gpu_logprobs import DT, check, make
from tests.test_gpu_timeout import short_waits

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
