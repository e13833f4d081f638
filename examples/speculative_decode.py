"""Speculative decoding with a small random keyless model: drafted trees are verified in one pass.

Two layers of keyless attention (Hq query heads over Hkv value heads, one W^R per value head) over paged
value-only caches, an embedding and the same matrix as the output layer. A draft model that is right some
of the time proposes a tree of tokens for every sequence; each step

1. appends the tree's value rows behind the committed ones   ``kl_append_v_chunk``
2. attends for the whole tree at once                         ``kl_tree_attention``
3. reads the greedy token and the drafts' log probabilities   ``kl_token_logprobs``
4. keeps the rows of the path that agrees with them           ``kl_tree_commit``

and so produces the tokens of one-by-one greedy decoding (``kl_decode_step``) in fewer steps:

    python examples/speculative_decode.py
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_21848_gb300 as kl  # noqa: E402

LAYERS, VOCAB, WIDTH, HQ, HKV, D, PAGE = 2, 500, 256, 8, 2, 128, 16


class Model:
    """Random weights. The dense parts run in float64, so that both ways of decoding round the same
    queries and value rows to bf16."""

    def __init__(self, seed=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, std: (torch.randn(*s, generator=g, dtype=torch.float64) * std).to(device)  # noqa: E731
        self.embed = r(VOCAB, WIDTH, std=1.0)
        self.wq = [r(WIDTH, HQ * D, std=WIDTH ** -0.5) for _ in range(LAYERS)]
        self.wv = [r(WIDTH, HKV * D, std=WIDTH ** -0.5) for _ in range(LAYERS)]
        self.wo = [r(HQ * D, WIDTH, std=2.0 * (HQ * D) ** -0.5) for _ in range(LAYERS)]
        self.w_r = [r(HKV, D, D, std=D ** -0.5).to(torch.bfloat16) for _ in range(LAYERS)]

    def qv(self, layer, x):
        q, v = x @ self.wq[layer], x @ self.wv[layer]
        return q.view(-1, HQ, D).to(torch.bfloat16), v.view(-1, HKV, D).to(torch.bfloat16)

    def add(self, layer, x, o):
        x = x + o.double().reshape(-1, HQ * D) @ self.wo[layer]
        return x / x.norm(dim=-1, keepdim=True) * WIDTH ** 0.5

    def logits(self, x):
        return (x @ self.embed.t() * (4.0 / WIDTH ** 0.5)).float()


class Caches:
    """One value-only cache per layer with the same page table."""

    def __init__(self, batch, tokens, device="cuda"):
        per = -(-tokens // PAGE)
        ids = torch.randperm(batch * per, generator=torch.Generator().manual_seed(1)).to(torch.int32)
        self.table = ids.view(batch, per).to(device)
        self.v = [torch.zeros(batch * per, HKV, PAGE, D, dtype=torch.bfloat16, device=device) for _ in range(LAYERS)]
        self.shape = kl.make_shape(batch, HQ, HKV, D, PAGE, batch * per, per)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)


def greedy(model, first, steps):
    """[batch][steps] tokens, one by one."""
    B = first.numel()
    c = Caches(B, steps + 1)
    ws = torch.zeros(max(256, kl.kl_decode_workspace_size(c.shape, 0)), dtype=torch.uint8, device="cuda")
    token, out = first, []
    o = torch.empty(B, HQ, D, device="cuda")
    for t in range(steps):
        x = model.embed[token]
        lens = torch.full((B,), t + 1, dtype=torch.int32, device="cuda")
        for layer in range(LAYERS):
            q, v = model.qv(layer, x)
            kl.kl_decode_step(c.shape, q, model.w_r[layer], v, lens - 1, c.v[layer], c.table, lens,
                              kl.decode_options(0), o, kl.KL_FP32, ws, c.err)
            x = model.add(layer, x, o)
        token = model.logits(x).argmax(-1)
        out.append(token)
    assert int(c.err) == 0
    return torch.stack(out, 1)


def draft_tree(guess, gen, depth, width):
    """A tree below the pending token (node 0): a chain of guesses, each with width - 1 siblings.
    Returns (tokens, parents) of one sequence as lists."""
    tokens, parents, at = [], [], 0
    for d in range(depth):
        tokens.append(int(guess[d]))
        parents.append(at)
        for _ in range(width - 1):
            tokens.append(int(torch.randint(VOCAB, (1,), generator=gen)))
            parents.append(at)
        at = len(tokens) - width + 1
    return tokens, parents


def speculative(model, first, steps, draft, depth=4, width=3, seed=0):
    """The same tokens with trees of 1 + depth * width nodes; draft(b, n, depth) guesses the tokens that
    follow the first n + 1 of sequence b. Returns (tokens, verification steps, sum of log probabilities)."""
    B, N = first.numel(), 1 + depth * width
    gen = torch.Generator().manual_seed(seed)
    c = Caches(B, steps + N + 1)
    cu = torch.arange(0, (B + 1) * N, N, dtype=torch.int32, device="cuda")
    ws = torch.zeros(max(256, kl.kl_tree_workspace_size(c.shape, B * N, N, 0),
                         kl.kl_logprobs_workspace_size(B * N, VOCAB, 1)), dtype=torch.uint8, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    o = torch.empty(B * N, HQ, D, device="cuda")
    best, best_lp = (torch.empty(B * N, 1, dtype=t, device="cuda") for t in (torch.int32, torch.float32))
    child_lp, entropy = torch.empty(B * N, width, device="cuda"), torch.empty(B * N, device="cuda")
    out, logprob, rounds = [[] for _ in range(B)], 0.0, 0
    pending = first.tolist()
    while min(len(t) for t in out) < steps:
        rounds += 1
        tokens, parents = [], []
        for b in range(B):
            t, p = draft_tree(draft(b, len(out[b]), depth), gen, depth, width)
            tokens += [pending[b]] + t
            parents += [-1] + p
        par = torch.tensor(parents, dtype=torch.int32, device="cuda")
        children = torch.full((B * N, width), -1, dtype=torch.int32)
        filled = [0] * (B * N)
        for i, p in enumerate(parents):
            if p >= 0:
                at = i // N * N + p
                children[at, filled[at]] = tokens[i]
                filled[at] += 1
        lens += N
        x = model.embed[torch.tensor(tokens, device="cuda")]
        for layer in range(LAYERS):
            q, v = model.qv(layer, x)
            kl.kl_append_v_chunk(c.shape, v, c.table, lens, cu, B * N, N, c.v[layer], c.err)
            kl.kl_tree_attention(c.shape, q, model.w_r[layer], c.v[layer], c.table, lens, cu, par, B * N, N, 0,
                                 o, kl.KL_FP32, ws, c.err)
            x = model.add(layer, x, o)
        logits = model.logits(x)
        kl.kl_token_logprobs(B * N, VOCAB, VOCAB, logits, kl.KL_FP32, 1.0, children.cuda(), width, 1, child_lp,
                             entropy, best_lp, best, ws, c.err)
        # follow the greedy token down the tree
        greedy_token, greedy_lp = best[:, 0].tolist(), best_lp[:, 0].tolist()
        paths, n = torch.full((B, N), -1, dtype=torch.int32), []
        for b in range(B):
            node, path = 0, [0]
            while True:
                want = greedy_token[b * N + node]
                if len(out[b]) < steps:
                    out[b].append(want)
                    logprob += greedy_lp[b * N + node]
                below = [i for i in range(N) if parents[b * N + i] == node and tokens[b * N + i] == want]
                if not below:
                    break
                node = below[0]
                path.append(node)
            pending[b] = want
            paths[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
            n.append(len(path))
        path, count = paths.cuda(), torch.tensor(n, dtype=torch.int32, device="cuda")
        kept = torch.empty_like(lens)
        for layer in range(LAYERS):
            kl.kl_tree_commit(c.shape, cu, path, count, N, c.table, lens, kept, c.v[layer], c.err)
        # (a sequence that is done decodes on from its last step: its rows do not matter any more)
        lens = torch.minimum(kept, torch.full_like(kept, steps + 1))
    assert int(c.err) == 0
    return torch.tensor(out, device="cuda"), rounds, logprob


def main(batch=4, steps=48):
    kl.build()
    kl.load()
    model = Model()
    first = torch.arange(batch, device="cuda") * 7 % VOCAB
    want = greedy(model, first, steps)
    gen = torch.Generator().manual_seed(2)

    def draft(b, n, depth):
        """A stand-in for a draft model: the right token three times out of four."""
        right = want[b, n:n + depth].tolist() + [0] * depth
        return [t if float(torch.rand(1, generator=gen)) < 0.75 else int(torch.randint(VOCAB, (1,), generator=gen))
                for t in right[:depth]]

    got, rounds, logprob = speculative(model, first, steps, draft)
    assert torch.equal(got, want), "speculative decoding gave other tokens"
    print(f"{batch} sequences, {steps} tokens each: {steps} decode steps or {rounds} verification steps, "
          f"sum of log probabilities {logprob:.2f}")
    return rounds


if __name__ == "__main__":
    main()
