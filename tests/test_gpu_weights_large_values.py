"""kl_attention_weights with cached values that are finite and have no finite fp16 form: outputs in blocks of 128 rows are
computed in fp16 and not finite where a position sees such a row, and the weights are those of its finite scores."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import attention, close, inputs, on, weigh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [2, 20, 40])
@pytest.mark.parametrize("L,back", [(200, 2), (200, 1), (200, 15), (200, 150), (3000, 2), (3000, 16), (70, 65)])
@pytest.mark.parametrize("value", [70000.0, -3e20])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weights_of_finite_scores(n, L, back, value, dtype):
    """The row stands `back` tokens before the end: new, seen by some of the new tokens, or old, seen by all of them."""
    kl.build()
    kl.load()
    x = inputs((L, 90), (n, n), 8, 2)
    t = L - back
    x["v_cache"][int(x["block_table"][0, t // 16]), :, t % 16, 7] = value
    g = on(x)
    old = torch.zeros(2, 2, max(L, 90), device="cuda")
    few = 4 * n <= 32
    out, new = weigh(g, old, 0.0, dtype, flags=kl.KL_FLAG_RANGE if dtype == torch.bfloat16 and not few else 0)
    want, added = attention(g)
    close(new[0, :, :L], added[0, :, :L])
    close(new[1, :, :90], added[1, :, :90])
    sees = torch.arange(L - n, L) >= t
    if dtype == torch.bfloat16 and not few:
        assert (~torch.isfinite(out[:n][sees])).any(-1).all() and torch.isfinite(out[:n][~sees]).all()
    else:
        assert torch.isfinite(out).all()
    close(out[:n][~sees], want[:n][~sees], dtype) if (~sees).any() else None


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("n", [2, 20])
def test_rows_that_are_not_finite_still_give_no_weights(bad, n):
    kl.build()
    kl.load()
    x = inputs((200, 90), (n, n), 8, 2)
    x["v_cache"][int(x["block_table"][0, 198 // 16]), :, 198 % 16] = bad
    for dtype in (torch.bfloat16, torch.float32):
        flags = kl.KL_FLAG_RANGE if dtype == torch.bfloat16 and n == 20 else 0
        _, new = weigh(on(x), torch.zeros(2, 2, 200, device="cuda"), 0.0, dtype, flags=flags)
        assert torch.isnan(new[0]).all()
        close(new[1, :, :90], attention(on(x))[1][1, :, :90])
