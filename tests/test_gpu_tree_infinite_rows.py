"""kl_tree_attention: an infinite value in a drafted row whose score is -inf for the drafts that see it. Its weight of 0
times infinity is NaN by the definition; it must not pass as a row that weighs nothing."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._verify import REL, tree_inputs, tree_reference
from tests.test_gpu_tree import run

pytestmark = pytest.mark.gpu

# With this scale -1 times scale log2 e is a sum of three negative bf16 terms, so that each of them gives -inf.
SCALE = 0.05011000111699104


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


@pytest.mark.parametrize("splits", [0, 4])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafts", [(4, 3), (8, 7), (40, 70)])
def test_an_infinite_value_against_a_negative_query(drafts, out, splits):
    x = tree_inputs((530 + drafts[0], 90 + drafts[1]), drafts, 8, 2, seed=5)
    x["q"][:, :, 5] = -1.0
    want = tree_reference(x, scale=SCALE, composed=True)
    cu, bad = x["cu_q"].tolist(), {0: 1, 1: 0}
    for b, i in bad.items():
        t = int(x["seq_lens"][b]) - drafts[b] + i
        x["v_cache"][int(x["block_table"][b, t // 16]), :, t % 16, 5] = math.inf
    flags = kl.KL_FLAG_RANGE if out == torch.bfloat16 and drafts[0] > 8 else 0
    got = run(x, out, splits=splits, scale=SCALE, composed=True, flags=flags)
    for b in range(2):
        for i in range(drafts[b]):
            j = i
            while j > bad[b]:
                j = int(x["parents"][cu[b] + j])
            r = cu[b] + i
            if j == bad[b]:
                assert torch.isnan(got[r].float()).all(), (b, i)
            else:
                d = got[r].double() - want[r]
                assert float(d.norm() / want[r].norm()) < 4 * REL[out], (b, i)
