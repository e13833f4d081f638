"""kl_tree_attention: what its operands may cost, with bounds derived from them: the routed query as two terms
(three with fp32 outputs), cached values that are small."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._verify import tree_inputs, tree_reference
from tests.test_gpu_tree import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def two_tokens(n, seed):
    """Every draft weighs two cached tokens against each other whose scores of about 300 lie 0 to 6 apart (scale 1, a
    query dimension for each); all other tokens score 0 and weigh nothing."""
    x = tree_inputs((700 + n, 300 + n), (n, n // 2), 8, 2, seed=seed)
    g = torch.Generator().manual_seed(seed)
    T = x["q"].shape[0]
    x["q"] = torch.zeros_like(x["q"])
    x["q"][:, :, 0] = (2 * torch.randint(128, 200, (T, 8), generator=g)).to(torch.bfloat16)
    x["q"][:, :, 1] = (x["q"][:, :, 0].float() + 2 * torch.randint(-3, 4, (T, 8), generator=g)).to(torch.bfloat16)
    x["w_r"] = torch.eye(128, dtype=torch.bfloat16).expand_as(x["w_r"]).contiguous()
    x["v_cache"][..., :2] = 0
    for b, (s, t) in enumerate(((30, 601), (200, 7))):
        for at, dim in ((s, 0), (t, 1)):
            x["v_cache"][int(x["block_table"][b, at // 16]), :, at % 16, dim] = 1
    return x


@pytest.mark.parametrize("composed", [False, True])
@pytest.mark.parametrize("n", [20, 64, 128])
def test_large_scores_with_bf16_outputs(n, composed):
    # A score in units of log2 is below 600, and the second term of a query element leaves at most 2^-18 of it:
    # two scores are off by 2 x 600 x 2^-18 ln 2 at most, the weight of one of two tokens by a quarter of that, the
    # output by this times their distance, at most twice sqrt 2 of the result's norm for independent rows. fp16
    # weights add 2^-12 and the output's rounding, at rms over 128 dims, less than 2^-9.
    x = two_tokens(n, n)
    want = tree_reference(x, scale=1.0, composed=composed)
    d = run(x, torch.bfloat16, scale=1.0, composed=composed).double() - want
    bound = 2 * 600 * 2.0 ** -18 * 0.6932 / 4 * 2 * 2 ** 0.5 + 2.0 ** -12 + 2.0 ** -9
    assert float((d.norm(dim=-1) / want.norm(dim=-1)).max()) <= bound


@pytest.mark.parametrize("composed", [False, True])
def test_large_scores_with_fp32_outputs(composed):
    # Three terms leave at most 2^-24 of a score of up to 600 (in units of log2), and the eight steps of its leading
    # product truncate at most 2^-14 each; two scores, and the way to the output as above. (Two terms would leave
    # 2^-18 of 600.)
    x = two_tokens(40, 3)
    want = tree_reference(x, scale=1.0, composed=composed)
    d = run(x, torch.float32, scale=1.0, composed=composed).double() - want
    bound = 2 * (600 * 2.0 ** -24 + 8 * 2.0 ** -14) * 0.6932 / 4 * 2 * 2 ** 0.5
    assert float((d.norm(dim=-1) / want.norm(dim=-1)).max()) <= bound


@pytest.mark.parametrize("size", [2.0 ** -10, 2.0 ** -16])
def test_small_cached_values(size):
    # With bf16 outputs more than 32 rows take cached values in fp16: exactly from 2^-14 on, and within 2^-25 below.
    # The rest of the bound: the output's rounding (half a unit of 2^-7), and weights off by 2^-12 each, independently.
    x = tree_inputs((500, 140), (20, 64), 8, 2, seed=6)
    x["v_cache"] = (x["v_cache"].float() * size).to(torch.bfloat16)
    x["q"] = (x["q"].float() / size).to(torch.bfloat16)
    want = tree_reference(x)
    d = (run(x, torch.bfloat16).double() - want).abs()
    assert bool((d <= 2.0 ** -25 + 2.0 ** -8 * want.abs() + 2.0 ** -11 * want.abs().amax(-1, keepdim=True)).all())


@pytest.mark.parametrize("size", [2.0 ** -10, 2.0 ** -16, 2.0 ** -30])
@pytest.mark.parametrize("drafts", [(20, 64), (4, 2)])
def test_small_cached_values_with_fp32_outputs(size, drafts):
    x = tree_inputs((500, 140), drafts, 8, 2, seed=6)
    x["v_cache"] = (x["v_cache"].float() * size).to(torch.bfloat16)
    x["q"] = (x["q"].float() / size).to(torch.bfloat16)
    want = tree_reference(x)
    d = run(x, torch.float32).double() - want
    assert float(d.norm() / want.norm()) < 2e-6
