"""Waits of the window attention and the attention weights that run out (on purpose, by a limit of 1 ns): the call
returns with its flag, and the next one with a workspace filled with zeros again is right."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import KL, attention, close, inputs, on, shape_of, workspace
from tests.test_gpu_timeout import short_waits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("splits", [1, 3])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
def test_waits_run_out_and_the_next_call_is_right(weigh, splits, out):
    kl.build()
    kl.load()
    g = on(inputs((5000, 3000), (1, 2), 16, 2, 16))
    sh = shape_of(g)
    size = kl.kl_weights_workspace_size(sh, 3, 2, 5000, splits) if weigh else kl.kl_window_workspace_size(sh, 3, 2, 4000, 4, splits)
    ws, o = workspace(size), torch.full(g["q"].shape, float("nan"), dtype=out, device="cuda")
    err, new = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, 2, 5000, device="cuda")

    def call():
        if weigh:
            kl.kl_attention_weights(sh, g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"], 3, 2,
                                    None, 5000, 0.0, new, splits, o, KL[out], ws, err)
        else:
            kl.kl_window_attention(sh, g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"], 3, 2,
                                   4000, 4, splits, o, KL[out], ws, err)
        torch.cuda.synchronize()

    with short_waits(1):
        call()
    assert int(err) & kl.KL_FLAG_TIMEOUT
    ws.zero_()
    err.zero_()
    call()
    assert int(err) == 0
    want, added = attention(g) if weigh else attention(g, 4000, 4)
    close(o, want, out)
    if weigh:
        close(new[0], added[0])
        close(new[1, :, :3000], added[1, :, :3000])
