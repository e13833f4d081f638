"""kl_window_workspace_size is 0 for bad arguments alone, also where a call needs no workspace (CPU only)."""
from __future__ import annotations

import pytest

import paper_2606_21848_gb300 as kl
from tests.test_bounded_host import built, shape  # noqa: F401


@pytest.mark.parametrize("kw, max_q", [({}, 9), ({}, 512), (dict(num_q_heads=256), 1), (dict(wr_per_query_head=True), 33),
                                       (dict(num_q_heads=256), 4096), (dict(num_seqs=0), 512)])
def test_blocks_of_128_rows(kw, max_q):
    def size(total=2 * max_q, W=100, S=4, splits=0, **more):
        return kl.kl_window_workspace_size(shape(**dict(kw, **more)), total, max_q, W, S, splits)

    assert size() > 0
    for bad in (dict(num_kv_heads=3), dict(total=-1), dict(W=0), dict(S=-1), dict(splits=-1), dict(splits=1 << 20)):
        assert size(**bad) == 0, bad
