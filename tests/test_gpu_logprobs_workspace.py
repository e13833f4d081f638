"""The workspace of kl_token_logprobs: its size serves either type of logits."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests.test_gpu_logprobs import DT, check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("T,V", [(50, 36868), (9, 204804), (8, 233476), (50, 55300)])
def test_the_size_serves_both_types(T, V, dtype):
    # (sizes at which, on 152 SMs, rows of bf16 logits are cut into more chunks than rows of fp32 logits)
    x, t, _ = make(T, V, dtype, T)
    check(x, t, 8)                        # a workspace of exactly the size asked for


def test_more_rows_than_the_front_region_has_counters():
    # Rows that are cut between CTAs are joined through counters in the workspace, which other calls use as well.
    ws = torch.zeros(1 << 23, dtype=torch.uint8, device="cuda")
    T, V, top = 20000, 16400, 4
    x = torch.randn(T, V, generator=torch.Generator("cuda").manual_seed(1), device="cuda").mul_(3).to(torch.bfloat16)
    tok = torch.arange(T, dtype=torch.int32, device="cuda").mul_(7).remainder_(V).view(T, 1)
    for _ in range(2):
        y, t, _ = make(96, 50257, torch.float32)
        check(y, t, 20, ws=ws)
        lp, en, tl = (torch.full((T, k), 7.0, device="cuda") for k in (1, 1, top))
        ti = torch.full((T, top), 7, dtype=torch.int32, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        kl.kl_token_logprobs(T, V, V, x, kl.KL_BF16, 1.0, tok, 1, top, lp, en, tl, ti, ws, err)
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        for r in range(0, T, 2000):
            want = torch.log_softmax(x[r:r + 2000].double(), -1)
            # (the tolerance of test_gpu_logprobs)
            for got, ref in ((lp, want.gather(1, tok[r:r + 2000].long())),
                             (en, -(want.exp() * want).sum(-1, keepdim=True)),
                             (tl, want.gather(1, ti[r:r + 2000].long().clamp(0, V - 1)))):
                assert bool(((got[r:r + 2000].double() - ref).abs() <= 2.0 ** -20 * ref.abs().clamp_min(1) * 2).all()), r
            assert torch.equal(tl[r:r + 2000], tl[r:r + 2000].sort(-1, descending=True)[0])
            assert bool((tl[r:r + 2000, 0].double() - want.max(-1)[0]).abs().max() < 1e-4)
