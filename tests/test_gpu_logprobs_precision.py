"""kl_token_logprobs: the error of log probabilities does not grow with what a row held before its largest logit."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._verify import logprob_reference
from tests.test_gpu_logprobs import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


@pytest.mark.parametrize("dtype, V, low, high", [(torch.float32, 20000, 10.0, 11.0), (torch.bfloat16, 40000, 10.7, 11.5)])
def test_a_late_logit_that_dominates(dtype, V, low, high):
    # One row per CTA, in three chunks; in the last of them one logit holds at least half of the weight. With
    # z = 1 + tail, tail <= 1.1 relative to it: the tail's independent roundings leave z within 2^-24 to 2^-23,
    # log2 z <= 1.1 is within one unit of 2^-23, so its log probability is within
    # (2^-24 + 2^-23 ln 2 + 2^-25) < 2^-22, where the sums do not lose their roundings against the one large term.
    # (A reference that stays behind leaves log2 z near 14, whose rounding alone is up to 2^-21 ln 2.)
    T = 456
    g = torch.Generator().manual_seed(3)
    x = (torch.randn(T, V, generator=g) * 0.5).to(dtype)
    at = V - 1 - torch.randint(0, V // 6, (T,), generator=g)
    x[torch.arange(T), at] = torch.linspace(low, high, T).to(dtype)
    lp, en, tl, ti = run(x, at.view(T, 1), 2)
    a, b, c, d = logprob_reference(x, 1.0, at.view(T, 1), 2)
    assert torch.equal(ti, d)
    assert float((lp.double() - a).abs().max()) <= 2.0 ** -22
    assert float((tl[:, 0].double() - c[:, 0]).abs().max()) <= 2.0 ** -22
