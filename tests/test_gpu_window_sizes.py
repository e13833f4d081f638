"""Window attention of as many sequences as a grid has, and of more: a batch in blocks of 128 rows is refused before
anything is launched, one with few rows is computed."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import KL, attention, close, inputs, on, workspace

pytestmark = pytest.mark.gpu


def batch(B, n):
    """Two sequences with new tokens, at the ends of a batch of B; the others have none."""
    x = inputs((300, 77), (n, n))
    pages = x["block_table"].shape[1]
    table = torch.full((B, pages), -1, dtype=torch.int32)
    table[0], table[-1] = x["block_table"][0], x["block_table"][1]
    lens = torch.zeros(B, dtype=torch.int32)
    lens[0], lens[-1] = 300, 77
    cu = torch.full((B + 1,), n, dtype=torch.int32)
    cu[0], cu[-1] = 0, 2 * n
    want = attention(x, 100, 4)[0]
    return dict(on(x), block_table=table.cuda(), seq_lens=lens.cuda(), cu_q=cu.cuda()), want


def call(g, B, n, dtype):
    pages, Hkv, P, D = g["v_cache"].shape
    sh = kl.make_shape(B, g["q"].shape[1], Hkv, D, P, pages, g["block_table"].shape[1])
    out, err = torch.zeros(g["q"].shape, dtype=dtype, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = workspace(kl.kl_window_workspace_size(sh, 2 * n, n, 100, 4, 0))
    kl.kl_window_attention(sh, g["q"], g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"], g["cu_q"], 2 * n, n, 100, 4,
                           0, out, KL[dtype], ws, err)
    torch.cuda.synchronize()
    assert int(err) == 0
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sequences_of_a_grid(dtype):
    kl.build()
    kl.load()
    for B, n in ((65536, 40), (70000, 9)):
        g, _ = batch(B, n)
        with pytest.raises(kl.KLError) as e:
            call(g, B, n, dtype)
        assert e.value.status == kl.KL_ERR_UNSUPPORTED
    for B, n in ((65535, 40), (65536, 1), (70000, 8)):
        g, want = batch(B, n)
        close(call(g, B, n, dtype), want, dtype)
