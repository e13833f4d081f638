"""kl_tree_attention: what lengths do beside the tested sizes. A length past the block table is reported whatever the
sequence's number of drafts; a table much wider than the sequences changes no result."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._verify import tree_inputs, tree_reference
from tests.test_gpu_tree import check, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [(4, 0, 3), (8, 0, 7), (40, 0, 20)])
def test_a_length_past_the_table_without_drafts(drafts, out):
    x = tree_inputs((300, 100, 90), drafts, 8, 2)
    want = tree_reference(x)
    y = dict(x, seq_lens=x["seq_lens"].clone())
    y["seq_lens"][1] = x["block_table"].shape[1] * 16 + 1
    check(run(y, out, flags=kl.KL_FLAG_BAD_LENGTH), want, out)


@pytest.mark.parametrize("splits", [0, 3])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [(4, 2, 1), (8, 7, 0), (40, 64, 1)])
def test_a_table_much_wider_than_the_sequences(drafts, out, splits):
    x = tree_inputs((1500, 260, 40), drafts, 8, 2, seed=3)
    want = tree_reference(x)
    y = dict(x, block_table=torch.nn.functional.pad(x["block_table"], (0, 31 * x["block_table"].shape[1]), value=-1))
    check(run(y, out, splits=splits), want, out)


def test_a_wide_table_and_many_sequences():
    lens = tuple(60 + 37 * (i % 11) for i in range(90))
    x = tree_inputs(lens, tuple(1 + i % 4 for i in range(90)), 8, 2, seed=4)
    want = tree_reference(x)
    y = dict(x, block_table=torch.nn.functional.pad(x["block_table"], (0, 2000), value=-1))
    check(run(y), want)
    check(run(y, torch.bfloat16), want, torch.bfloat16)
