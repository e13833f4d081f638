"""Inputs and 64-bit references of the verification operators (tree attention, log probabilities, commit),
written from their definitions on the CPU, apart from the library."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests._inputs import tiny

# Tree attention, relative to the 2-norm of the result. The routed query and the softmax weights are sums of
# two bf16 operands (relative error at most 2^-17 each); a score is a sum of 128 products with independent
# errors, so it is off by about 2^-17 of its own size, and scores here are a few units: weights, and with
# them the output, are off by a few 2^-17 at most. bf16 outputs add half a unit of 2^-8.
REL = {torch.float32: 2e-5, torch.bfloat16: 2.0 ** -9 + 2e-5}


def make_parents(kind, n, gen):
    if kind == "chain":
        return [i - 1 for i in range(n)]
    if kind == "star":
        return [-1] * n
    if kind == "binary":
        return [(i - 1) // 2 if i else -1 for i in range(n)]
    return [int(torch.randint(-1, i, (1,), generator=gen)) if i else -1 for i in range(n)]   # "random"


def tree_inputs(lens, drafts, Hq=8, Hkv=2, P=16, kind="random", seed=5, wr_per_query_head=False, table="permuted"):
    """Sequences of lens[b] cached rows, the last drafts[b] of them a tree."""
    assert all(0 <= n <= L for n, L in zip(drafts, lens))
    x = tiny(len(lens), Hq, Hkv, 128, P, tuple(lens), seed, table, wr_per_query_head)
    gen = torch.Generator().manual_seed(seed + 31)
    T = int(sum(drafts))
    x["q"] = torch.randn(T, Hq, 128, generator=gen).to(torch.bfloat16)
    x["cu_q"] = torch.tensor(np.concatenate([[0], np.cumsum(drafts)]), dtype=torch.int32)
    x["parents"] = torch.tensor([p for n in drafts for p in make_parents(kind, n, gen)], dtype=torch.int32)
    x["drafts"] = list(drafts)
    x["wr_per_query_head"] = wr_per_query_head
    return x


def rows_of(x, b):
    """Sequence b's cached rows in order, [Hkv][L][D] in 64 bits."""
    P, L = x["v_cache"].shape[2], int(x["seq_lens"][b])
    ids = x["block_table"][b, :-(-L // P)].long()
    r = x["v_cache"][ids].double().transpose(0, 1)
    return r.reshape(r.shape[0], -1, r.shape[-1])[:, :L]


def visible(parents, L, n):
    """[n][L]: what each draft sees."""
    see = torch.zeros(n, L, dtype=torch.bool)
    see[:, :L - n] = True
    for i in range(n):
        j = i
        while j >= 0:
            see[i, L - n + j] = True
            j = int(parents[j])
    return see


def tree_reference(x, scale=None, composed=False):
    T, Hq, D = x["q"].shape
    Hkv = x["v_cache"].shape[1]
    q = x["q"].double()
    if not composed:
        w = x["w_r"].double()
        q = torch.einsum("thk,hkj->thj", q, w if x["wr_per_query_head"] else w.repeat_interleave(Hq // Hkv, 0))
    out = torch.zeros(T, Hq, D, dtype=torch.float64)
    cu = x["cu_q"].tolist()
    for b, L in enumerate(x["seq_lens"].tolist()):
        n = cu[b + 1] - cu[b]
        if n == 0:
            continue
        v = rows_of(x, b).repeat_interleave(Hq // Hkv, 0)
        s = torch.einsum("nhd,htd->hnt", q[cu[b]:cu[b + 1]], v) * (scale or 1 / math.sqrt(D))
        see = visible(x["parents"][cu[b]:cu[b + 1]], L, n)
        p = torch.softmax(s.masked_fill(~see, -math.inf), -1)
        # (a row that a draft does not see takes no part, whatever it holds)
        vv = torch.where(see.any(0)[None, :, None], v, 0.0)
        if not torch.isfinite(vv).all():
            o = torch.stack([torch.einsum("ht,htd->hd", p[:, i, see[i]], v[:, see[i]]) for i in range(n)])
        else:
            o = torch.einsum("hnt,htd->nhd", p, vv)
        out[cu[b]:cu[b + 1]] = o
    return out


def logprob_reference(logits, scale, tokens, top):
    """(logprobs, entropy, top_logprobs, top_ids) in 64 bits; scale as the float32 it is passed as."""
    x = logits.double() * float(np.float32(scale))
    lp = torch.log_softmax(x, -1)
    none = torch.isinf(x).all(-1) & (x < 0).all(-1)
    lp = torch.where(none[:, None], -math.inf, lp)
    ent = -torch.where(lp == -math.inf, 0.0, lp.exp() * lp).sum(-1)
    got = torch.gather(lp, 1, tokens.long().clamp_min(0))
    got = torch.where(tokens < 0, 0.0, got)
    ids = torch.argsort(logits.double(), dim=-1, descending=True, stable=True)[:, :top]
    return got, ent, torch.gather(lp, 1, ids), ids.to(torch.int32)
