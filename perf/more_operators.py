"""A value-only cache that stays bounded while a stream goes on, as cases that can be timed and compared.

A server that serves long streams either lets each token see a window of the last tokens and a few first
ones, or keeps account of the attention that each cached row receives and evicts the rows with the least.
Three operators:

- ``window``   ``kl_window_attention``: attention of new tokens (one per sequence, a chunk or a whole
               prompt) to the last ``window`` tokens and the first ``sinks`` ones;
- ``weights``  ``kl_attention_weights``: causal attention of a sequence's last tokens that also adds
               up the softmax weight that each cached row receives;
- ``evict``    ``kl_evict``: the rows with the largest accumulated weights stay and move together.

``own`` false: the same in elementary torch operations in 32 bits. Head layouts, page sizes and lengths
are those of this package's own workloads and of the ranges around them; windows and budgets are generic.
"""
import math

import torch

own = False

# --------------------------------------------------------------------------------- cases ----
# window, weights: sequences, query and value heads, head dim 128, cached tokens len_lo .. len_hi (the new
# ones included), new tokens per sequence new_lo .. new_hi, page size, W^R ("kv": per value head, "q": per
# query head, "none": the query is already composed), output type, split count (0: the library chooses).
# window: the window and the first tokens that stay visible; weights: what old weights are multiplied by.
# evict: budget of rows per value head, first and last rows that always stay, in place or to other pages.
_SEQ = dict(page=16, wr="kv", out="bf16", splits=0)


def _attend(op, name, seqs, q_heads, kv_heads, len_lo, len_hi, new_lo, new_hi, **more):
    c = dict(_SEQ, op=op, seqs=seqs, q_heads=q_heads, kv_heads=kv_heads, len_lo=len_lo, len_hi=len_hi,
             new_lo=new_lo, new_hi=new_hi)
    c.update(more)
    return dict(c, name=name) if name else c


def _evict(name, seqs, kv_heads, head_dim, len_lo, len_hi, budget, sinks, recent, page=16, in_place=True):
    c = dict(op="evict", seqs=seqs, kv_heads=kv_heads, head_dim=head_dim, len_lo=len_lo, len_hi=len_hi,
             budget=budget, sinks=sinks, recent=recent, page=page, in_place=in_place)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one user's next token with a short window: launch and latency
        _attend("window", "window_one", 1, 32, 8, 2999, 2999, 1, 1, window=1000, sinks=4),
        # the next tokens of a full batch of a 70B-class GQA model
        _attend("window", "window_70b", 128, 64, 8, 8192, 8192, 1, 1, window=4096, sinks=64, page=32),
        # a serving batch of mixed lengths, one to four tokens each, 32-bit outputs
        _attend("window", "window_ragged_fp32", 64, 32, 8, 512, 32768, 1, 4, window=2047, sinks=5, out="fp32"),
        # chunks of prompts that are read in pieces
        _attend("window", "window_chunk", 8, 32, 8, 8192, 8192, 512, 512, window=1024, sinks=4),
        # a whole prompt, one W^R per query head, groups of 6 query heads
        _attend("window", "window_prompt", 1, 12, 2, 32768, 32768, 32768, 32768, window=4096, sinks=64, wr="q"),
        # one user's next token, weights in 32 bits: latency
        _attend("weights", "weights_one", 1, 32, 8, 2000, 2000, 1, 1, decay=1.0, out="fp32"),
        # the next tokens of a batch, every row's weight added up
        _attend("weights", "weights_batch", 64, 64, 8, 8192, 8192, 1, 1, decay=1.0, page=32),
        # mixed lengths, weights that fade
        _attend("weights", "weights_ragged", 24, 32, 8, 301, 20011, 1, 1, decay=0.96875),
        # behind a prompt: the weights that its last 16 tokens give
        _attend("weights", "weights_prompt", 4, 32, 8, 4001, 6007, 16, 16, decay=0.0),
        # a few streams that have grown past their budget
        _evict("evict_small", 8, 8, 128, 2100, 2304, 2048, 4, 256),
        # one long prompt cut down to an eighth, to pages of its own
        _evict("evict_long", 1, 8, 128, 131072, 131072, 16384, 4, 1024, in_place=False),
        # a batch cut down to half
        _evict("evict_batch", 64, 8, 128, 8192, 8192, 4096, 64, 512, page=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "window", "weights", "weights", "evict", "evict"])
    page = rng.choice([16, 16, 32, 64, 128])
    if op == "evict":
        hkv, d = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128, 128])
        seqs, longest = _log(rng, 1, 128), _log(rng, 64, 131072)
        longest = max(64, min(longest, (1 << 29) // (hkv * 2 * d * seqs)))    # at most half a GiB of rows
        budget = max(8, int(longest * rng.uniform(0.05, 0.98)))
        sinks, recent = rng.choice([0, 1, 4, 64]), rng.choice([0, 1, 32, 200])
        sinks = min(sinks, budget // 4)
        return _evict(None, seqs, hkv, d, rng.randint(longest // 2, longest), longest, budget, sinks,
                      min(recent, budget // 4), page, rng.random() < 0.7)
    hq, hkv = rng.choice([(32, 8), (64, 8), (12, 2), (28, 4), (32, 1), (8, 8), (128, 8), (16, 16)])
    new = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 2048 if op == "window" else 32)])
    seqs, longest = _log(rng, 1, 128), _log(rng, 64, 65536)
    more = dict(page=page, wr=rng.choice(["kv", "kv", "q", "none"]), out=rng.choice(["bf16", "bf16", "fp32"]),
                splits=rng.choice([0, 0, 0, rng.randint(1, 32)]))
    if op == "window":
        more.update(window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 5, 64, 130]))
        seen = min(longest, more["window"] + more["sinks"] + min(new, 256))
    else:
        more.update(decay=rng.choice([0.0, 0.5, 0.96875, 1.0]))
        seen = longest
    # at most 1 GiB of cached rows, and 2^28 scores
    seqs = max(1, min(seqs, (1 << 28) // (hq * new * seen)))
    longest = max(new, min(longest, (1 << 30) // (hkv * 256 * seqs)))
    lo = longest if rng.random() < 0.5 else rng.randint(new, longest)
    return _attend(op, None, seqs, hq, hkv, lo, longest, rng.randint(1, new), new, **more)


# -------------------------------------------------------------------------------- inputs ----
def _spread(n, lo, hi):
    """n whole numbers spread evenly over lo .. hi."""
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _randn(shape, g, std=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)
    return x if std == 1.0 else x * std


def _table(need, perm):
    """Block table of sequences of `need` pages, the pages in the order of perm (-1 past a sequence's)."""
    col = torch.arange(int(need.max()), device="cuda")
    at = ((torch.cumsum(need, 0) - need)[:, None] + col[None, :]).clamp_max(perm.numel() - 1)
    return torch.where(col[None, :] < need[:, None], perm[at], -1).to(torch.int32).contiguous()


def _shuffled(values, seed):
    t = torch.tensor(values, dtype=torch.int64)
    return t[torch.randperm(len(values), generator=torch.Generator().manual_seed(seed))].cuda()


def _inputs(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, D, P, Hkv = c["seqs"], c.get("head_dim", 128), c["page"], c["kv_heads"]
    s = dict(op=c["op"])
    lens = _shuffled(_spread(B, c["len_lo"], c["len_hi"]), seed)
    need = (lens + P - 1) // P
    pages, extra = int(need.sum()), 0
    if c["op"] == "evict" and not c["in_place"]:
        need_to = (lens.clamp_max(c["budget"]) + P - 1) // P
        extra = int(need_to.sum())
    # a shuffled page pool that holds the sequences (and the pages that evicted ones move to)
    perm = torch.randperm(pages + extra, generator=g, device="cuda").to(torch.int32)
    s.update(table=_table(need, perm[:pages]), pages=pages + extra, lens=lens.to(torch.int32))
    s["v"] = _randn((pages + extra, Hkv, P, D), g)
    most = int(lens.max())
    if c["op"] != "window":
        # weights added up so far: many small ones, a few large ones, some rows that nothing looked at
        u = torch.rand((B, Hkv, most), generator=g, device="cuda")
        w = (-torch.log(u.clamp_min(1e-7))) ** 4 * 0.05
        w = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.03, 0.0, w)
        seen = lens if c["op"] == "evict" else lens - 1
        s["weights"] = torch.where(torch.arange(most, device="cuda") < seen[:, None, None], w, 0.0).contiguous()
        s["new_weights"] = torch.zeros_like(s["weights"])
    if c["op"] == "evict":
        s["to"] = s["table"] if c["in_place"] else _table(need_to, perm[pages:])
        if s["to"].shape[1] < s["table"].shape[1]:
            s["to"] = torch.nn.functional.pad(s["to"], (0, s["table"].shape[1] - s["to"].shape[1]), value=-1)
        s["kept"] = torch.full((B, Hkv, c["budget"]), -1, dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.zeros_like(s["lens"])
        s.update(budget=c["budget"], sinks=c["sinks"], recent=c["recent"])
        return s
    n = torch.minimum(_shuffled(_spread(B, c["new_lo"], c["new_hi"]), seed + 1), lens)
    T, Hq = int(n.sum()), c["q_heads"]
    s.update(q=_randn((T, Hq, D), g), w_r=None, rows=T, max_q=c["new_hi"], splits=c["splits"],
             dtype=torch.float32 if c["out"] == "fp32" else torch.bfloat16)
    if c["wr"] != "none":
        s["w_r"] = _randn((Hq if c["wr"] == "q" else Hkv, D, D), g, D ** -0.5)
    s["cu"] = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), torch.cumsum(n, 0)]).to(torch.int32)
    s.update(window=c.get("window", most), sinks=c.get("sinks", 0), decay=c.get("decay", 0.0))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _keep(case, s)
    return s


def _keep(c, s):
    """What a program that uses the library keeps between calls: shape, outputs, workspace, error word."""
    from paper_2606_21848_gb300 import _lib
    Hkv = c["kv_heads"]
    s["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["shape"] = _lib.make_shape(c["seqs"], c.get("q_heads", Hkv), Hkv, c.get("head_dim", 128), c["page"],
                                 s["pages"], s["table"].shape[1], c.get("wr") == "q")
    if c["op"] == "evict":
        ws = _lib.kl_evict_workspace_size(s["shape"], s["weights"].shape[2], c["budget"])
        s["ws"] = torch.zeros(max(256, ws), dtype=torch.uint8, device="cuda")
        return
    s["out"] = torch.zeros(s["q"].shape, device="cuda", dtype=s["dtype"])
    s["kl_dtype"] = _lib.KL_FP32 if c["out"] == "fp32" else _lib.KL_BF16
    if c["op"] == "window":
        ws = _lib.kl_window_workspace_size(s["shape"], s["rows"], s["max_q"], s["window"], s["sinks"], s["splits"])
    else:
        ws = _lib.kl_weights_workspace_size(s["shape"], s["rows"], s["max_q"], s["weights"].shape[2], s["splits"])
    s["ws"] = torch.zeros(max(256, ws), dtype=torch.uint8, device="cuda")


# ----------------------------------------------------------------------------- the passes ----
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2606_21848_gb300 import _lib
    if s["op"] == "window":
        _lib.kl_window_attention(s["shape"], s["q"], s["w_r"], s["v"], s["table"], s["lens"], s["cu"], s["rows"],
                                 s["max_q"], s["window"], s["sinks"], s["splits"], s["out"], s["kl_dtype"],
                                 s["ws"], s["err"])
        return s["out"]
    if s["op"] == "weights":
        _lib.kl_attention_weights(s["shape"], s["q"], s["w_r"], s["v"], s["table"], s["lens"], s["cu"], s["rows"],
                                  s["max_q"], s["weights"], s["weights"].shape[2], s["decay"], s["new_weights"],
                                  s["splits"], s["out"], s["kl_dtype"], s["ws"], s["err"])
        return s["out"], s["new_weights"]
    _lib.kl_evict(s["shape"], s["weights"], s["weights"].shape[2], s["budget"], s["sinks"], s["recent"],
                  s["table"], s["lens"], s["to"], s["v"], s["new_weights"], s["kept"], s["new_lens"], s["ws"], s["err"])
    return s["kept"], s["new_lens"], s["new_weights"], s["v"].view(torch.int16)


def _run_plain(s):
    return {"window": _plain_window, "weights": _plain_weights, "evict": _plain_evict}[s["op"]](s)


def _routed(s, Hq):
    q = s["q"].float()
    if s["w_r"] is not None:
        w = s["w_r"].float().repeat_interleave(Hq // s["w_r"].shape[0], 0)
        q = torch.matmul(q.transpose(0, 1), w).transpose(0, 1)
    return q


def _plain_window(s):
    (T, Hq, D), (B, _), (_, Hkv, P, _) = s["q"].shape, s["table"].shape, s["v"].shape
    G, W, S, lens, cu = Hq // Hkv, s["window"], s["sinks"], s["lens"].long(), s["cu"].long()
    # blocks of up to 256 rows of a sequence, each with the tokens that one of its rows may see
    N = min(256, s["max_q"])
    M = -(-s["max_q"] // N)
    n, at = cu[1:] - cu[:-1], torch.arange(M * N, device="cuda").view(M, N)
    row = (cu[:-1, None, None] + at).clamp_max(T - 1).view(B * M, N)
    live = (at < n[:, None, None]).view(B * M, N)
    pos = ((lens - n)[:, None, None] + at).view(B * M, N)
    last = lens.repeat_interleave(M)[:, None]
    tok = torch.cat([torch.arange(S, device="cuda").expand(B * M, S),
                     pos[:, :1] - (W - 1) + torch.arange(W + N - 1, device="cuda")], 1)
    there = (tok >= 0) & (tok < last)
    there[:, S:] &= tok[:, S:] >= S
    t = torch.where(there, tok, 0)
    page = torch.gather(s["table"].long().repeat_interleave(M, 0), 1, t // P).clamp_min(0)
    x = torch.where(there[:, :, None, None], s["v"][page, :, t % P].float(), 0.0).transpose(1, 2)  # [., Hkv, K, D]
    q = _routed(s, Hq)[row].reshape(B * M, N, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B * M, Hkv, G * N, D)
    p = (torch.matmul(q, x.transpose(2, 3)) * D ** -0.5).reshape(B * M, Hkv, G, N, -1)
    see = there[:, None, :] & (tok[:, None, :] <= pos[:, :, None])
    see &= (tok[:, None, :] < S) | (tok[:, None, :] > pos[:, :, None] - W)
    p = p.masked_fill_(~see[:, None, None], -math.inf)
    p = torch.exp_(p.sub_(p.amax(-1, keepdim=True)))
    o = torch.matmul(p.reshape(B * M, Hkv, G * N, -1), x) / p.sum(-1).reshape(B * M, Hkv, G * N, 1)
    o = o.reshape(B * M, Hkv, G, N, D).permute(0, 3, 1, 2, 4).reshape(B * M, N, Hq, D)
    out = torch.zeros((T + 1, Hq, D), device="cuda")
    return out.index_copy_(0, torch.where(live, row, T).reshape(-1), o.reshape(-1, Hq, D))[:T].to(s["dtype"])


def _plain_weights(s):
    (T, Hq, D), (B, C), (_, Hkv, P, _) = s["q"].shape, s["table"].shape, s["v"].shape
    G, N, lens, cu = Hq // Hkv, s["max_q"], s["lens"].long(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), n, output_size=T)
    i = torch.arange(T, device="cuda") - cu[seq]
    x = s["v"][s["table"].long().clamp_min(0)].permute(0, 2, 1, 3, 4).reshape(B, Hkv, C * P, D).float()
    q = torch.zeros((B, N, Hq, D), device="cuda").index_put_((seq, i), _routed(s, Hq))
    q = q.reshape(B, N, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * N, D)
    p = (torch.matmul(q, x.transpose(2, 3)) * D ** -0.5).reshape(B, Hkv, G, N, C * P)
    d = torch.arange(N, device="cuda")
    t = torch.arange(C * P, device="cuda")
    see = t[None, None, :] <= ((lens - n)[:, None] + d)[:, :, None]                    # [B, N, tokens]
    p = p.masked_fill_(~see[:, None, None], -math.inf)
    p = torch.exp_(p.sub_(p.amax(-1, keepdim=True)))
    p = p.div_(p.sum(-1, keepdim=True))
    o = torch.matmul(p.reshape(B, Hkv, G * N, C * P), x).reshape(B, Hkv, G, N, D).permute(0, 3, 1, 2, 4)
    p = p.mul_((d < n[:, None])[:, None, None, :, None]).sum((2, 3))                   # [B, Hkv, tokens]
    E = s["weights"].shape[2]
    new = s["decay"] * s["weights"] + p[:, :, :E]
    new = torch.where(torch.arange(E, device="cuda") < lens[:, None, None], new, s["new_weights"])
    return o.reshape(B, N, Hq, D)[seq, i].to(s["dtype"]), new


def _plain_evict(s):
    w, P, K = s["weights"], s["v"].shape[2], s["budget"]
    (B, Hkv, E), L = w.shape, s["lens"].long()[:, None, None]
    t = torch.arange(E, device="cuda")
    # whole numbers in the order of the weights (none is negative), ties to the lowest index; rows that always stay first
    order = w.contiguous().view(torch.int32).long() * (1 << 24) - t
    order = torch.where((t < s["sinks"]) | (t >= L - s["recent"]), (1 << 62) - t, order)
    order = torch.where(t < L, order, -(1 << 62) - t)
    k = min(K, E)
    ids = torch.topk(order, k, -1).indices
    ids = torch.sort(ids, -1).values
    new_len = L.clamp_max(K)
    j = torch.arange(k, device="cuda")
    live = (j < new_len).expand(B, Hkv, k)
    kept = s["kept"].clone()
    kept[:, :, :k] = torch.where(live, ids, -1).to(torch.int32)
    new = torch.where(t < L, 0.0, s["new_weights"])
    new[:, :, :k] = torch.where(live, torch.gather(w, 2, ids), new[:, :, :k])
    b, g, at = torch.nonzero(live, as_tuple=True)
    src, v = ids[b, g, at], s["v"]
    rows = v[s["table"].long()[b, src // P], g, src % P]
    v[s["to"].long()[b, at // P], g, at % P] = rows
    return kept, new_len[:, 0, 0].to(torch.int32), new, v.view(torch.int16)


# ----------------------------------------------------------------------------------- work ----
def work(case):
    c = case
    B, Hkv, D = c["seqs"], c["kv_heads"], c.get("head_dim", 128)
    lens = _spread(B, c["len_lo"], c["len_hi"])
    if c["op"] == "evict":
        # a sequence within its budget stays where it is, unless it moves to other pages; the rows behind the
        # first that always stay move, whichever are chosen
        rows = sum(min(n, c["budget"]) - (min(n, c["sinks"]) if c["in_place"] else 0)
                   for n in lens if n > c["budget"] or not c["in_place"])
        ids = sum(min(n, c["budget"]) for n in lens)
        return {"bytes": float(Hkv * (4 * D * rows + 4 * ids + 8 * sum(lens)) + 12 * B), "flops": 0.0}
    Hq = c["q_heads"]
    n = _spread(B, c["new_lo"], c["new_hi"])
    # lengths and new tokens are shuffled apart: their products by the means
    T, mean_len, mean_new = sum(n), sum(lens) / B, sum(n) / B
    if c["op"] == "window":
        tokens = sum(min(x, c["window"] + c["sinks"] + mean_new - 1) for x in lens)
        # row i of a chunk at position p sees min(p + 1, window + sinks) tokens
        full = c["window"] + c["sinks"]
        first = mean_len - mean_new + 1
        low = min(max(full - first, 0.0), mean_new)
        pairs = B * (low * (first + first + low) / 2 + (mean_new - low) * min(full, mean_len))
    else:
        tokens = sum(lens)
        pairs = T * (mean_len - (mean_new - 1) / 2)
    hw = {"q": Hq, "kv": Hkv, "none": 0}[c["wr"]]
    nbytes = (tokens * Hkv * D * 2 + hw * D * D * 2 + T * Hq * D * (2 + (4 if c["out"] == "fp32" else 2))
              + tokens / c["page"] * 4 + 12 * B + (8 * Hkv * tokens if c["op"] == "weights" else 0))
    return {"bytes": float(nbytes), "flops": 4.0 * Hq * D * pairs + (2.0 * T * Hq * D * D if hw else 0.0)}


# ---------------------------------------------------------------------------------- exact ----
def exact(case, seed):
    """The outputs in 64 bits, from the definitions, sequence by sequence."""
    c = case
    if c["op"] == "evict":
        return None                                     # choices and copies
    s = _inputs(c, seed)
    Hq, Hkv, P, D = c["q_heads"], c["kv_heads"], c["page"], 128
    G = Hq // Hkv
    q = s["q"].double()
    if s["w_r"] is not None:
        w = s["w_r"].double()
        q = torch.einsum("thk,hkj->thj", q, w if c["wr"] == "q" else w.repeat_interleave(G, 0))
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    new = s["new_weights"].double() if c["op"] == "weights" else None
    cu = s["cu"].tolist()
    for b, L in enumerate(s["lens"].tolist()):
        rows = s["v"][s["table"][b, :-(-L // P)].long()].double().transpose(0, 1).reshape(Hkv, -1, D)[:, :L]
        n, total = cu[b + 1] - cu[b], 0.0
        for i in range(0, n, 512):
            m = min(512, n - i)
            p = torch.arange(L - n + i, L - n + i + m, device="cuda")[:, None]
            if c["op"] == "window":
                first = max(0, L - n + i - c["window"] + 1)
                t = torch.cat([torch.arange(min(c["sinks"], first), device="cuda"),
                               torch.arange(first, L - n + i + m, device="cuda")])
                hidden = (t > p) | ((t >= c["sinks"]) & (t <= p - c["window"]))
            else:
                t = torch.arange(L, device="cuda")
                hidden = t > p
            v = rows[:, t]
            qb = q[cu[b] + i:cu[b] + i + m].reshape(m, Hkv, G, D).permute(1, 2, 0, 3)
            a = torch.softmax((torch.einsum("hgnd,htd->hgnt", qb, v) / math.sqrt(D)).masked_fill(hidden, -math.inf), -1)
            out[cu[b] + i:cu[b] + i + m] = torch.einsum("hgnt,htd->nhgd", a, v).reshape(m, Hq, D)
            if new is not None:
                total = total + a.sum((1, 2))
        if new is not None:
            new[b, :, :L] = c["decay"] * s["weights"][b, :, :L].double() + total
    return out if new is None else (out, new)
