"""Split counts beyond the states that one CTA merges, on one long sequence of one value head."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import attention, close, inputs, on, weigh, window

pytestmark = pytest.mark.gpu
L = 131072


@pytest.fixture(scope="module", params=[16, 32])
def case(request):
    kl.build()
    kl.load()
    g = on(inputs((L,), (1,), request.param, 1, 128))
    return g, attention(g)


@pytest.mark.parametrize("splits", [255, 256, 257, 400, 512, 1024])
def test_window(case, splits):
    g, (want, _) = case
    for dtype in (torch.bfloat16, torch.float32):
        close(window(g, L, 0, dtype, splits), want, dtype)


@pytest.mark.parametrize("splits", [256, 512, 1024])
def test_weights(case, splits):
    g, (want, added) = case
    for dtype in (torch.bfloat16, torch.float32):
        out, new = weigh(g, torch.zeros(1, 1, L, device="cuda"), 0.0, dtype, splits)
        close(out, want, dtype)
        close(new, added)
