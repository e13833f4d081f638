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
