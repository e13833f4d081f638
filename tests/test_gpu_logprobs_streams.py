"""kl_token_logprobs where every CTA streams several chunks: the ring of copies is refilled, its barriers go through
several phases, candidates are kept over chunks, cut when the list fills up and taken again where a later chunk
overflows it, and rows begin and end inside a CTA's run.

Tolerance: that of test_gpu_logprobs (2^-20 of the size of the result, at least of 1). A thread's sum has up to 600 terms
and keeps about sqrt(600) 2^-25 of it; 256 of them and the parts of a row join with their roundings kept."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._verify import logprob_reference
from tests.test_gpu_logprobs import DT, close, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def rows(T, V, dtype, seed):
    """Rows of nine kinds in turn."""
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(T, V, generator=g, device="cuda") * 3
    up = torch.arange(V, device="cuda", dtype=torch.float32)
    x[1::9] = up / 64                                      # rising: every chunk holds all of the largest
    x[2::9] = -up / 64
    x[3::9] = 1.5                                          # ties everywhere
    x[4::9] = torch.randint(0, 3, x[4::9].shape, generator=g, device="cuda").float()
    x[5::9] = torch.where(torch.rand(x[5::9].shape, generator=g, device="cuda") < 2e-4, x[5::9], -math.inf)
    x[6::9] = torch.where(torch.rand(x[6::9].shape, generator=g, device="cuda") < 2e-4, x[6::9], torch.finfo(dtype).min)
    x[7::9, -1] = 30.0
    x[7::9, V // 2:V // 2 + 50] = 29.0
    x[8::9] = torch.floor(up / 3000)                       # rising steps of equal logits
    x = x.to(dtype)
    if T > 14:
        x[14] = -math.inf
    return x, torch.randint(0, V, (T, 3), generator=g, device="cuda")


@pytest.mark.parametrize("start", [0, 3])
@pytest.mark.parametrize("top", [0, 8, 32])
@pytest.mark.parametrize("T,V", [(460, 100003), (1500, 33001), (5000, 9001)])
@pytest.mark.parametrize("dtype", DT)
def test_several_chunks_per_cta(dtype, T, V, top, start):
    x, t = rows(T, V, dtype, top)
    lp, en, tl, ti = run(x, t, top, 0.7, start=start)
    for r in range(0, T, 500):
        s = slice(r, r + 500)
        a, b, c, d = (y.cpu() for y in logprob_reference(x[s], 0.7, t[s], top))
        # (scale times the lowest value overflows fp32: weight 0 and a log probability of -inf)
        a, c = (torch.where(y < -1e30, -math.inf, y) for y in (a, c))
        got_a, got_c = (torch.where(y < -1e30, -math.inf, y) for y in (lp[s], tl[s]))
        size = lambda y: torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y)).clamp_min(1.0)  # noqa: E731
        close(got_a, a, size(a))
        close(en[s], b, size(b) * 2)
        assert torch.equal(ti[s], d)
        close(got_c, c, size(c))
