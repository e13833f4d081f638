"""The verification step's operators together: speculative decoding of a small random model gives the tokens of
greedy decoding, in fewer steps (examples/speculative_decode.py)."""
from __future__ import annotations

import importlib.util
import os

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests.conftest import ROOT

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("speculative_decode",
                                                  os.path.join(ROOT, "examples", "speculative_decode.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    kl.build()
    kl.load()
    return m


def test_the_example(example):
    assert example.main() < 30


@pytest.mark.parametrize("depth,width", [(1, 1), (6, 1), (2, 5), (7, 4)])
def test_trees_of_other_shapes(example, depth, width):
    model = example.Model(seed=depth)
    first = torch.tensor([3, 141], device="cuda")
    want = example.greedy(model, first, 30)
    gen = torch.Generator().manual_seed(depth)

    def draft(b, n, d):
        right = want[b, n:n + d].tolist() + [0] * d
        return [t if float(torch.rand(1, generator=gen)) < 0.6 else 1 for t in right[:d]]

    got, rounds, logprob = example.speculative(model, first, 30, draft, depth, width, seed=width)
    assert torch.equal(got, want)
    assert rounds <= 30 and logprob < 0
