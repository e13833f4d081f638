"""The verification step of speculative decoding over a paged value-only cache, as cases that can be
timed and compared.

A server that drafts several continuations of every sequence appends the drafted tokens' value rows,
attends for all of them at once, reads the model's logits for them, and keeps the accepted path. Three
operators:

- ``tree``      ``kl_tree_attention``: attention of a tree of drafted tokens over the cache; a draft
                sees the committed tokens, itself and its ancestors;
- ``logprobs``  ``kl_token_logprobs``: log probabilities of given tokens, the entropy and the largest
                logits of each row of logits;
- ``commit``    ``kl_tree_commit``: the rows of the accepted path move to where decoding goes on.

``own`` false: the same in elementary torch operations in 32 bits. Head layouts, page sizes and lengths
are those of this package's own workloads and of the ranges around them; vocabularies are generic.
"""
import math

import torch

own = False

# --------------------------------------------------------------------------------- cases ----
# tree: sequences, query and value heads, head dim 128, cached tokens len_lo .. len_hi (drafts
# included), drafts per sequence drafts_lo .. drafts_hi, shape of the trees ("chain": one path, "wide":
# random parents, "star": every draft follows the last committed token), page size, W^R ("kv": per
# value head, "q": per query head, "none": the query is already composed), output type, split count
# (0: the library chooses), fraction of cached values scaled by 20.
_TREE = dict(page=16, tree="wide", wr="kv", out="bf16", splits=0, outliers=0.0)


def _tree(name, seqs, q_heads, kv_heads, len_lo, len_hi, drafts_lo, drafts_hi, **more):
    c = dict(_TREE, op="tree", seqs=seqs, q_heads=q_heads, kv_heads=kv_heads, len_lo=len_lo,
             len_hi=len_hi, drafts_lo=drafts_lo, drafts_hi=drafts_hi)
    c.update(more)
    return dict(c, name=name) if name else c


def _logprobs(name, rows, vocab, dtype, tokens, top, pad=0, scale=1.0):
    c = dict(op="logprobs", rows=rows, vocab=vocab, dtype=dtype, tokens=tokens, top=top, pad=pad,
             scale=scale)
    return dict(c, name=name) if name else c


def _commit(name, seqs, kv_heads, head_dim, len_lo, len_hi, drafts, page):
    c = dict(op="commit", seqs=seqs, kv_heads=kv_heads, head_dim=head_dim, len_lo=len_lo,
             len_hi=len_hi, drafts=drafts, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user, a short context, four drafted tokens in a row: launch and latency
        _tree("tree_chain4", 1, 32, 8, 700, 700, 4, 4, tree="chain"),
        # interactive serving: a few sequences, small trees
        _tree("tree_small_batch", 8, 32, 8, 4096, 4096, 8, 8),
        # one long document, a wide tree: the cache is cut over the whole GPU
        _tree("tree_long", 1, 32, 8, 131072, 131072, 32, 32, tree="wide"),
        # a serving batch of mixed lengths and mixed tree sizes, outlier values
        _tree("tree_ragged", 64, 32, 8, 512, 32768, 1, 24, outliers=0.01),
        # a full batch of a 70B-class GQA model
        _tree("tree_70b", 64, 64, 8, 8192, 8192, 16, 16, page=32),
        # large trees, one W^R per query head, groups of 6 query heads, fp32 output
        _tree("tree_group6_fp32", 12, 12, 2, 3001, 6007, 61, 64, wr="q", out="fp32"),
        # one row of logits with its alternatives: latency
        _logprobs("logprobs_one", 1, 32000, "bf16", 1, 5),
        # the drafted tokens of a serving batch, an odd vocabulary whose rows are not 16-byte aligned
        _logprobs("logprobs_odd_fp32", 96, 50257, "fp32", 3, 20, scale=1.25),
        _logprobs("logprobs_batch", 512, 128256, "bf16", 4, 8),
        # the whole batch's trees, scored without alternatives
        _logprobs("logprobs_large", 2048, 151936, "bf16", 1, 0),
        # after a verification step: the accepted rows of a few sequences, and of a full batch
        _commit("commit_small", 8, 8, 128, 4096, 4096, 8, 16),
        _commit("commit_70b", 256, 8, 128, 2048, 8192, 32, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree"] * 5 + ["logprobs"] * 3 + ["commit"])
    if op == "logprobs":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        rows, vocab = _log(rng, 1, 4096), _log(rng, 1000, 262144)
        rows = max(1, min(rows, int(6e8 / (vocab * (2 if dtype == "bf16" else 4)))))
        return _logprobs(None, rows, vocab, dtype, rng.choice([1, 1, 2, 4, 8]),
                         rng.choice([0, 1, 5, 8, 20, 32]), rng.choice([0, 0, 1, 8, 13]),
                         rng.choice([1.0, 1.0, 0.5, 1.6]))
    if op == "commit":
        return _commit(None, _log(rng, 1, 256), rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128]),
                       200, _log(rng, 256, 4096), rng.randint(1, 64), rng.choice([16, 32, 64, 128]))
    hq, hkv = rng.choice([(32, 8), (64, 8), (12, 2), (28, 4), (32, 1), (8, 8), (128, 8), (16, 16)])
    seqs, drafts = _log(rng, 1, 128), _log(rng, 1, 64)
    longest = _log(rng, 64, 131072)
    # at most 1 GiB of cached rows, and 2^29 scores
    longest = min(longest, (1 << 30) // (hkv * 256 * seqs), (1 << 29) // (seqs * hq * drafts))
    longest = max(longest, drafts)
    lo = longest if rng.random() < 0.5 else rng.randint(drafts, longest)
    return _tree(None, seqs, hq, hkv, lo, longest, rng.randint(1, drafts), drafts,
                 tree=rng.choice(["chain", "wide", "wide", "star"]), page=rng.choice([16, 16, 32, 64, 128]),
                 wr=rng.choice(["kv", "kv", "q", "none"]), out=rng.choice(["bf16", "bf16", "fp32"]),
                 splits=rng.choice([0, 0, 0, rng.randint(1, 32)]), outliers=rng.choice([0.0, 0.0, 0.01]))


# -------------------------------------------------------------------------------- inputs ----
def _spread(n, lo, hi):
    """n whole numbers spread evenly over lo .. hi."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _randn(shape, g, std=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    return x if std == 1.0 else x * std


def _pool(lens, kv_heads, page, head_dim, g):
    """A shuffled page pool that holds `lens`, and its block table (-1 past a sequence's pages)."""
    need = (lens + page - 1) // page
    pages = int(need.sum())
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    col = torch.arange(int(need.max()), device="cuda")
    at = ((torch.cumsum(need, 0) - need)[:, None] + col[None, :]).clamp_max(pages - 1)
    table = torch.where(col[None, :] < need[:, None], perm[at], -1).to(torch.int32).contiguous()
    return _randn((pages, kv_heads, page, head_dim), g), table, pages


def _shuffled(values, seed):
    t = torch.tensor(values, dtype=torch.int64)
    return t[torch.randperm(len(values), generator=torch.Generator().manual_seed(seed))].cuda()


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(op=c["op"])
    if c["op"] == "logprobs":
        T, V = c["rows"], c["vocab"]
        x = torch.randn((T, V + c["pad"]), generator=g, device="cuda", dtype=torch.float32) * 3.0
        x = x.to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
        tokens = torch.randint(0, V, (T, c["tokens"]), generator=g, device="cuda").to(torch.int32)
        # the first given token of most rows is a likely one
        likely = x[:, :V].argmax(-1).to(torch.int32)
        keep = torch.rand(T, generator=g, device="cuda") < 0.7
        tokens[:, 0] = torch.where(keep, likely, tokens[:, 0])
        s.update(logits=x, tokens=tokens, vocab=V, top=c["top"], scale=c["scale"])
        return s
    B, D, P = c["seqs"], c.get("head_dim", 128), c["page"]
    lens = _shuffled(_spread(B, c["len_lo"], c["len_hi"]), seed)
    s["v"], s["table"], s["pages"] = _pool(lens, c["kv_heads"], P, D, g)
    if c["op"] == "commit":
        n = torch.minimum(lens, torch.full_like(lens, c["drafts"]))
        # the accepted path: a random increasing choice of drafts, mostly short
        u = torch.rand((B, c["drafts"]), generator=g, device="cuda")
        there = torch.arange(c["drafts"], device="cuda")[None, :] < n[:, None]
        pick = (u < torch.rand((B, 1), generator=g, device="cuda") * 0.5) & there
        path = torch.sort(torch.where(pick, torch.arange(c["drafts"], device="cuda")[None, :], 1 << 20), -1).values
        s["counts"] = pick.sum(-1).to(torch.int32)
        s["path"] = torch.where(path < (1 << 20), path, -1).to(torch.int32).contiguous()
    else:
        n = _shuffled(_spread(B, c["drafts_lo"], c["drafts_hi"]), seed + 1)
        n = torch.minimum(n, lens)
        T, Hq = int(n.sum()), c["q_heads"]
        if c["outliers"]:
            s["v"] = torch.where(torch.rand(s["v"].shape, generator=g, device="cuda") < c["outliers"],
                                 s["v"] * 20, s["v"])
        i = torch.arange(T, device="cuda") - torch.repeat_interleave(torch.cumsum(n, 0) - n, n)
        if c["tree"] == "chain":
            parents = i - 1
        elif c["tree"] == "star":
            parents = torch.full_like(i, -1)
        else:       # a random earlier draft or the root, later drafts mostly deeper
            u = torch.rand(T, generator=g, device="cuda")
            parents = torch.minimum((u.sqrt() * (i + 1).float()).long(), i) - 1
        s.update(parents=parents.to(torch.int32), q=_randn((T, Hq, D), g), w_r=None, rows=T,
                 max_q=c["drafts_hi"], splits=c["splits"],
                 dtype=torch.float32 if c["out"] == "fp32" else torch.bfloat16)
        if c["wr"] != "none":
            s["w_r"] = _randn((Hq if c["wr"] == "q" else c["kv_heads"], D, D), g, D ** -0.5)
    s["lens"] = lens.to(torch.int32)
    s["cu"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cumsum(n, 0)]).to(torch.int32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _keep(case, s)
    return s


def _keep(c, s):
    """What a program that uses the library keeps between calls: shape, outputs, workspace, error word."""
    from paper_2606_21848_gb300 import _lib
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if c["op"] == "logprobs":
        T, K = c["rows"], c["top"]
        f = dict(device="cuda", dtype=torch.float32)
        s["logp"], s["entropy"] = torch.zeros((T, c["tokens"]), **f), torch.zeros(T, **f)
        s["top_logp"], s["top_ids"] = torch.zeros((T, K), **f), torch.zeros((T, K), device="cuda", dtype=torch.int32)
        s["kl_dtype"] = _lib.KL_BF16 if c["dtype"] == "bf16" else _lib.KL_FP32
        ws = _lib.kl_logprobs_workspace_size(T, c["vocab"], K)
    else:
        P, D = c["page"], c.get("head_dim", 128)
        s["shape"] = _lib.make_shape(c["seqs"], c.get("q_heads", c["kv_heads"]), c["kv_heads"], D, P,
                                     s["pages"], s["table"].shape[1], c.get("wr") == "q")
        ws = 0
    if c["op"] == "commit":
        s["new_lens"] = torch.zeros_like(s["lens"])
    if c["op"] == "tree":
        s["out"] = torch.zeros(s["q"].shape, device="cuda", dtype=s["dtype"])
        s["kl_dtype"] = _lib.KL_FP32 if c["out"] == "fp32" else _lib.KL_BF16
        ws = _lib.kl_tree_workspace_size(s["shape"], s["rows"], s["max_q"], c["splits"])
    s["ws"] = torch.zeros(max(256, ws), dtype=torch.uint8, device="cuda")


# ----------------------------------------------------------------------------- the passes ----
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2606_21848_gb300 import _lib
    if s["op"] == "tree":
        _lib.kl_tree_attention(s["shape"], s["q"], s["w_r"], s["v"], s["table"], s["lens"], s["cu"],
                               s["parents"], s["rows"], s["max_q"], s["splits"], s["out"], s["kl_dtype"],
                               s["ws"], s["err"])
        return s["out"]
    if s["op"] == "logprobs":
        _lib.kl_token_logprobs(s["logits"].shape[0], s["vocab"], s["logits"].shape[1], s["logits"],
                               s["kl_dtype"], s["scale"], s["tokens"], s["tokens"].shape[1], s["top"],
                               s["logp"], s["entropy"], s["top_logp"], s["top_ids"], s["ws"], s["err"])
        return (s["logp"], s["entropy"]) + ((s["top_logp"], s["top_ids"]) if s["top"] else ())
    _lib.kl_tree_commit(s["shape"], s["cu"], s["path"], s["counts"], s["path"].shape[1], s["table"],
                        s["lens"], s["new_lens"], s["v"], s["err"])
    return s["v"].view(torch.int16), s["new_lens"]


def _run_plain(s):
    return {"tree": _plain_tree, "logprobs": _plain_logprobs, "commit": _plain_commit}[s["op"]](s)


def _plain_tree(s):
    q, table, lens, cu = s["q"].float(), s["table"].long().clamp_min(0), s["lens"].long(), s["cu"].long()
    (T, Hq, D), (B, W), (_, Hkv, P, _) = q.shape, table.shape, s["v"].shape
    n, G, N = cu[1:] - cu[:-1], Hq // Hkv, s["max_q"]
    if s["w_r"] is not None:
        w = s["w_r"].float().repeat_interleave(Hq // s["w_r"].shape[0], 0)
        q = torch.matmul(q.transpose(0, 1), w).transpose(0, 1)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), n, output_size=T)
    i = torch.arange(T, device="cuda") - cu[seq]
    # the drafts of every sequence, padded to N, and who is whose ancestor
    qp = torch.zeros((B, N, Hq, D), device="cuda").index_put_((seq, i), q)
    par = torch.zeros((B, N, N + 1), device="cuda").index_put_((seq, i, s["parents"].long() + 1), torch.ones(T, device="cuda"))
    seen = torch.linalg.matrix_power(torch.eye(N, device="cuda") + par[:, :, 1:], N) > 0
    x = s["v"][table].permute(0, 2, 1, 3, 4).reshape(B, Hkv, W * P, D).float()
    qp = qp.view(B, N, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, D)
    p = torch.matmul(qp, x.transpose(2, 3)).view(B, Hkv, G, N, W * P) * D ** -0.5
    d = torch.arange(W * P, device="cuda")[None, :] - (lens - n)[:, None]              # [B, tokens]
    draft = torch.gather(seen, 2, d.clamp(0, N - 1)[:, None, :].expand(B, N, W * P))
    see = torch.where(d[:, None, :] < 0, True, draft & (d < n[:, None])[:, None, :])
    p = p.masked_fill_(~see[:, None, None], -math.inf)
    p = torch.exp_(p.sub_(p.amax(-1, keepdim=True)))
    o = torch.matmul(p.view(B, Hkv, G * N, W * P), x) / p.sum(-1).view(B, Hkv, G * N, 1)
    o = o.view(B, Hkv, G, N, D).permute(0, 3, 1, 2, 4).reshape(B, N, Hq, D)
    return o[seq, i].to(s["dtype"])


def _order(x):
    """Whole numbers in the order of the logits, ties to the lowest index (all distinct)."""
    b = x.float().view(torch.int32).long() if x.dtype == torch.bfloat16 else x.contiguous().view(torch.int32).long()
    b = torch.where(b >= 0, b, -(b & 0x7FFFFFFF))
    return b * (1 << 32) - torch.arange(x.shape[1], device="cuda")


def _plain_logprobs(s):
    raw = s["logits"][:, :s["vocab"]]
    x = raw.float() * s["scale"]
    m = x.amax(-1, keepdim=True)
    x = x - m
    e = torch.exp(x)
    z = e.sum(-1, keepdim=True)
    lz = torch.log(z)
    logp = torch.gather(x, 1, s["tokens"].long()) - lz
    entropy = (lz - (e * x).sum(-1, keepdim=True) / z)[:, 0]
    if not s["top"]:
        return logp, entropy
    ids = torch.topk(_order(raw), s["top"], -1).indices
    return logp, entropy, torch.gather(x, 1, ids) - lz, ids.to(torch.int32)


def _plain_commit(s):
    v, P = s["v"], s["v"].shape[2]
    n = (s["cu"][1:] - s["cu"][:-1]).long()
    base = s["lens"].long() - n
    b, j = torch.nonzero(torch.arange(s["path"].shape[1], device="cuda")[None, :] < s["counts"][:, None], as_tuple=True)
    src, dst = base[b] + s["path"][b, j].long(), base[b] + j
    table = s["table"].long()
    v[table[b, dst // P], :, dst % P] = v[table[b, src // P], :, src % P]
    return v.view(torch.int16), (base + s["counts"]).to(torch.int32)


# ----------------------------------------------------------------------------------- work ----
def work(case):
    c = case
    if c["op"] == "logprobs":
        n = c["rows"] * c["vocab"]
        return {"bytes": float(n * (2 if c["dtype"] == "bf16" else 4) + c["rows"] * (8 * c["tokens"] + 8 * c["top"] + 4)),
                "flops": 6.0 * n}
    B = c["seqs"]
    lens = _spread(B, c["len_lo"], c["len_hi"])
    if c["op"] == "commit":
        # about a quarter of the drafts is accepted; the rows are read and written
        rows = sum(min(c["drafts"], n) for n in lens) / 4.0
        return {"bytes": 4.0 * rows * c["kv_heads"] * c["head_dim"] + 16.0 * B + 4.0 * rows, "flops": 0.0}
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], 128
    n = _spread(B, c["drafts_lo"], c["drafts_hi"])
    # lengths and drafts are shuffled apart: their products by the means, ancestors not counted
    T, tokens = sum(n), sum(lens)
    hw = {"q": Hq, "kv": Hkv, "none": 0}[c["wr"]]
    nbytes = (tokens * Hkv * D * 2 + hw * D * D * 2 + T * Hq * D * (2 + (4 if c["out"] == "fp32" else 2))
              + sum(-(-x // c["page"]) for x in lens) * 4 + 8 * B + 4 * T)
    flops = 4.0 * Hq * D * T * max(1.0, tokens / B - T / B) + (2.0 * T * Hq * D * D if hw else 0.0)
    return {"bytes": float(nbytes), "flops": flops}


# ---------------------------------------------------------------------------------- exact ----
def exact(case, seed):
    """The outputs in 64 bits, from the definitions, sequence by sequence and row by row."""
    c = case
    s = _inputs(c, seed)
    if c["op"] == "commit":
        return None                                     # copies
    if c["op"] == "logprobs":
        logp, ent, top = [], [], []
        for r in range(0, c["rows"], 64):
            raw = s["logits"][r:r + 64, :c["vocab"]].double()
            lp = torch.log_softmax(raw * s["scale"], -1)
            logp.append(torch.gather(lp, 1, s["tokens"][r:r + 64].long()))
            ent.append(-(lp.exp() * lp).sum(-1))
            if c["top"]:
                top.append(torch.sort(lp, -1, descending=True).values[:, :c["top"]])
        out = torch.cat(logp), torch.cat(ent)
        return out + (torch.cat(top), None) if c["top"] else out
    Hq, Hkv, P, D = c["q_heads"], c["kv_heads"], c["page"], 128
    G = Hq // Hkv
    q = s["q"].double()
    if s["w_r"] is not None:
        w = s["w_r"].double()
        q = torch.einsum("thk,hkj->thj", q, w if c["wr"] == "q" else w.repeat_interleave(G, 0))
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    cu, parents = s["cu"].tolist(), s["parents"].tolist()
    for b, L in enumerate(s["lens"].tolist()):
        n = cu[b + 1] - cu[b]
        rows = s["v"][s["table"][b, :-(-L // P)].long()].double().transpose(0, 1).reshape(Hkv, -1, D)[:, :L]
        hidden = torch.ones((n, L), dtype=torch.bool)
        hidden[:, :L - n] = False
        for i in range(n):
            j = i
            while j >= 0:
                hidden[i, L - n + j] = False
                j = parents[cu[b] + j]
        qb = q[cu[b]:cu[b + 1]].reshape(n, Hkv, G, D).permute(1, 2, 0, 3)
        sc = torch.einsum("hgnd,htd->hgnt", qb, rows) / math.sqrt(D)
        p = torch.softmax(sc.masked_fill(hidden.cuda(), -math.inf), -1)
        out[cu[b]:cu[b + 1]] = torch.einsum("hgnt,htd->nhgd", p, rows).reshape(n, Hq, D)
    return out
