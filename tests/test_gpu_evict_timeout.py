"""Waits of an eviction in place that run out (on purpose, by a limit of 1 ns): the call returns with its flag, and the
next one on a fresh cache, with the same workspace, is right."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import workspace
from tests.test_gpu_evict import case, reference
from tests.test_gpu_timeout import short_waits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,Hkv,D,budget", [((60000,), 1, 128, 40000), ((30000, 20000, 400), 2, 64, 19000),
                                               ((9000,) * 5, 8, 128, 8000)])
def test_waits_run_out_and_the_next_call_is_right(lens, Hkv, D, budget):
    kl.build()
    kl.load()
    c = case(lens, Hkv, D, 16, kind="random")
    B, _, E = c["w"].shape
    sh = kl.make_shape(B, Hkv, Hkv, D, 16, c["v"].shape[0], c["table"].shape[1])
    w, table = c["w"].cuda(), c["table"].cuda()
    seq, err = torch.tensor(c["lens"], dtype=torch.int32).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = workspace(kl.kl_evict_workspace_size(sh, E, budget))

    def call():
        v, new, new_lens = c["v"].cuda(), torch.zeros_like(w), torch.zeros_like(seq)
        kept = torch.zeros(B, Hkv, budget, dtype=torch.int32, device="cuda")
        kl.kl_evict(sh, w, E, budget, 4, 100, table, seq, table, v, new, kept, new_lens, ws, err)
        torch.cuda.synchronize()
        return v.cpu(), kept.cpu(), new_lens.tolist()

    with short_waits(1):
        call()
    assert int(err) == kl.KL_FLAG_TIMEOUT
    err.zero_()
    v, kept, new_lens = call()
    assert int(err) == 0 and not ws[:65536].any()
    for b, g, L, ids, rows in reference(c, budget, 4, 100):
        j = torch.arange(len(ids))
        assert new_lens[b] == len(ids) and kept[b, g, :len(ids)].tolist() == ids
        assert torch.equal(v[c["table"][b, j // 16].long(), g, j % 16], rows)
