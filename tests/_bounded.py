"""Inputs and 64-bit references of the operators of a bounded cache (window attention, attention weights,
eviction), written from their definitions, apart from the library."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2606_21848_gb300 as kl
from tests._inputs import tiny
from tests._verify import rows_of

# Relative to the 2-norm of the result.
# fp32 outputs, and weights: query and weights are sums of three bf16 terms (what is left is below 2^-25 of a value),
# the tensor core's sums of 128 products truncate at 2^-23 or so of the sum, as do a few fp32 additions: a score of a
# few units is off by some 2^-22 of the largest partial sum, and with it weights and outputs. 2e-5 is ten times that.
# bf16 outputs: two terms of the query (2^-17) or fp16 weights (2^-12 of a weight's share, independent from
# weight to weight), and half a unit of bf16 (2^-9 of a value at most).
REL = {torch.float32: 2e-5, torch.bfloat16: 2.0 ** -9 + 2.0 ** -12}


def inputs(lens, news, Hq=8, Hkv=2, P=16, seed=5, wr_per_query_head=False, table="permuted"):
    """Sequences of lens[b] cached rows, the last news[b] of them new tokens."""
    assert all(0 <= n <= L for n, L in zip(news, lens))
    x = tiny(len(lens), Hq, Hkv, 128, P, tuple(lens), seed, table, wr_per_query_head)
    gen = torch.Generator().manual_seed(seed + 31)
    T = int(sum(news))
    x["q"] = torch.randn(T, Hq, 128, generator=gen).to(torch.bfloat16)
    x["cu_q"] = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32)
    x["news"] = list(news)
    x["wr_per_query_head"] = wr_per_query_head
    return x


def visible(L, n, window, sinks, device="cpu"):
    """[n][L]: what each new token sees."""
    p = torch.arange(L - n, L, device=device)[:, None]
    t = torch.arange(L, device=device)
    return (t <= p) & ((t < sinks) | (t > p - window))


def attention(x, window=1 << 30, sinks=0, scale=None, composed=False):
    """(out [T][Hq][D], weights [B][Hkv][longest]) in 64 bits; a token that a row does not see takes no part."""
    T, Hq, D = x["q"].shape
    Hkv = x["v_cache"].shape[1]
    G, dev = Hq // Hkv, x["q"].device
    q = x["q"].double()
    if not composed:
        w = x["w_r"].double()
        q = torch.einsum("thk,hkj->thj", q, w if x["wr_per_query_head"] else w.repeat_interleave(G, 0))
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=dev)
    lens, cu = x["seq_lens"].tolist(), x["cu_q"].tolist()
    weights = torch.zeros(len(lens), Hkv, max(lens), dtype=torch.float64, device=dev)
    for b, L in enumerate(lens):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        see = visible(L, n, window, sinks, dev)
        any_sees = see.any(0)
        v = torch.where(any_sees[None, :, None], rows_of(x, b), 0.0)
        finite = torch.isfinite(v).all(0).all(-1)
        s = torch.einsum("nghd,gtd->gnht", q[cu[b]:cu[b + 1]].reshape(n, Hkv, G, D), v) * (scale or 1 / math.sqrt(D))
        a = torch.softmax(s.masked_fill(~see[None, :, None], -math.inf), -1)
        o = torch.einsum("gnht,gtd->ngh" + "d", a, torch.where(finite[None, :, None], v, 0.0)).reshape(n, Hq, D)
        o[(see & ~finite).any(-1)] = math.nan
        out[cu[b]:cu[b + 1]] = o
        weights[b, :, :L] = a.sum((1, 2))
    if x["q"].is_cuda:
        torch.cuda.synchronize()
    return out, weights


def keep(weights, L, budget, sinks, recent):
    """Ids of the rows that stay, of one value head's weights (a list of floats)."""
    if L <= budget:
        return list(range(L))
    middle = sorted(range(sinks, L - recent), key=lambda t: (-max(weights[t], 0.0) if weights[t] == weights[t] else 0.0, t))
    return sorted(list(range(sinks)) + middle[:budget - sinks - recent] + list(range(L - recent, L)))


def shape_of(x, B=None, scale=0.0):
    pages, Hkv, P, D = x["v_cache"].shape
    return kl.make_shape(B or len(x["news"]), x["q"].shape[1], Hkv, D, P, pages, x["block_table"].shape[1],
                         x["wr_per_query_head"], scale)


def on(x, device="cuda"):
    return {k: (v.to(device) if torch.is_tensor(v) else v) for k, v in x.items()}


KL = {torch.float32: kl.KL_FP32, torch.bfloat16: kl.KL_BF16}


def workspace(size):
    return torch.zeros(max(256, size), dtype=torch.uint8, device="cuda")


def window(g, W, S, dtype=torch.float32, splits=0, scale=0.0, composed=False, max_q=None, ws=None, flags=0, out=None,
           maybe=0):
    """kl_window_attention on device inputs; `maybe`: flags that may be raised as well."""
    T = g["q"].shape[0]
    sh = shape_of(g, scale=scale)
    max_q = max_q or max(1, max(g["news"]))
    out = torch.full(g["q"].shape, float("nan"), dtype=dtype, device="cuda") if out is None else out
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    need = kl.kl_window_workspace_size(sh, T, max_q, W, S, splits)
    ws = workspace(need) if ws is None else ws
    kl.kl_window_attention(sh, g["q"], None if composed else g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"],
                           g["cu_q"], T, max_q, W, S, splits, out, KL[dtype], ws, err)
    torch.cuda.synchronize()
    assert int(err.item()) & ~maybe == flags
    assert not ws[:65536].any()                        # counters are back at zero
    return out


def weigh(g, old, decay, dtype=torch.float32, splits=0, scale=0.0, composed=False, max_q=None, ws=None, flags=0,
          new=None):
    """kl_attention_weights on device inputs: (out, new weights)."""
    T = g["q"].shape[0]
    sh = shape_of(g, scale=scale)
    max_q = max_q or max(1, max(g["news"]))
    out = torch.full(g["q"].shape, float("nan"), dtype=dtype, device="cuda")
    new = torch.full_like(old, -7.0) if new is None else new
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    stride = old.shape[2]
    ws = workspace(kl.kl_weights_workspace_size(sh, T, max_q, stride, splits)) if ws is None else ws
    kl.kl_attention_weights(sh, g["q"], None if composed else g["w_r"], g["v_cache"], g["block_table"], g["seq_lens"],
                            g["cu_q"], T, max_q, old, stride, decay, new, splits, out, KL[dtype], ws, err)
    torch.cuda.synchronize()
    assert int(err.item()) == flags
    assert not ws[:65536].any()
    return out, new


def close(got, want, dtype=None):
    got = got.double().to(want.device)
    assert torch.isfinite(got).all()
    rel = float((got - want).norm()) / max(float(want.norm()), 1e-30)
    assert rel <= REL[dtype or torch.float32], rel
    assert float((got - want).abs().max()) <= 40 * REL[dtype or torch.float32] * max(float(want.abs().max()), 1e-30)
