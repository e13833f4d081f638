"""kl_token_logprobs against log_softmax in 64 bits: vocabularies around vectors and chunks, alignments, ties,
masked logits, rows that are masked whole, huge and lowest values, refusals of token ids.

Tolerance: fp32 sums of at most 2^18 terms in 3 levels (64 per thread, 256 threads, chunks), each rounding
2^-24; 2^x off by at most 2^-22 relative: log z within 2^-21, and x - log z within 2^-22 of its size."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._verify import logprob_reference

pytestmark = pytest.mark.gpu
DT = {torch.bfloat16: kl.KL_BF16, torch.float32: kl.KL_FP32}


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def run(logits, tokens, top, scale=1.0, start=0, flags=0, ws=None, vocab=None):
    """logits [T][V] on the CPU, placed `start` elements into a padded buffer."""
    T, V = logits.shape
    stride = V + 3
    buf = torch.full((start + T * stride + 16,), float("nan"), dtype=logits.dtype, device="cuda")
    view = buf[start:start + T * stride].view(T, stride)
    view[:, :V] = logits.cuda()
    tok = tokens.to(torch.int32).cuda().contiguous()
    K = tok.shape[1]
    lp = torch.full((T, K), 7.0, device="cuda")
    en = torch.full((T,), 7.0, device="cuda")
    tl = torch.full((T, top), 7.0, device="cuda")
    ti = torch.full((T, top), 7, dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    if ws is None:
        ws = torch.zeros(max(256, kl.kl_logprobs_workspace_size(T, V, top)), dtype=torch.uint8, device="cuda")
    kl.kl_token_logprobs(T, V, stride, view, DT[logits.dtype], scale, tok, K, top, lp, en, tl, ti, ws, err)
    torch.cuda.synchronize()
    assert int(err.item()) == flags
    assert not ws[:min(ws.numel(), 4 * T)].any() or ws.numel() < 65536
    return lp.cpu(), en.cpu(), tl.cpu(), ti.cpu()


def close(got, want, size):
    """|got - want| within 2^-20 of the row's largest |x| difference to log z (at least 1)."""
    same = (got.double() == want) | (torch.isnan(got) & torch.isnan(want))
    ok = same | ((got.double() - want).abs() <= 2.0 ** -20 * size)
    assert bool(ok.all()), float((got.double() - want).abs().max())


def check(logits, tokens, top, scale=1.0, **kw):
    lp, en, tl, ti = run(logits, tokens, top, scale, **kw)
    a, b, c, d = logprob_reference(logits, scale, tokens, top)
    size = lambda t: torch.where(torch.isfinite(t), t.abs(), torch.zeros_like(t)).clamp_min(1.0)  # noqa: E731
    close(lp, a, size(a))
    close(en, b, (size(b) * 2))
    assert torch.equal(ti, d)
    close(tl, c, size(c))


def make(T, V, dtype, seed=0, std=3.0):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(T, V, generator=g) * std).to(dtype)
    return x, torch.randint(0, V, (T, 3), generator=g), g


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 255, 1000, 2047, 8191, 8192, 8193, 16383, 16384, 16385, 16391,
                               32768, 50257, 131075])
def test_vocabularies(dtype, V):
    x, t, _ = make(3, V, dtype, V)
    for top in {0, 1, min(V, 5), min(V, 32)}:
        check(x, t, top)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("start", range(9))
def test_alignments(dtype, start):
    x, t, _ = make(5, 16390, dtype, start)
    check(x, t, 20, 0.7, start=start)


@pytest.mark.parametrize("dtype", DT)
def test_ties_go_to_the_lowest_index(dtype):
    x, t, g = make(6, 40000, dtype)
    x[0] = 1.5                                             # one value everywhere
    x[1] = torch.randint(0, 3, (40000,), generator=g).to(dtype)
    x[2, 7000:7040] = 30.0                                 # more equal largest than wanted
    x[3] = torch.where(x[3] > 0, 0.0, -0.0).to(dtype)      # zeros of both signs are equal
    x[4] = torch.arange(40000).to(dtype)                   # rising: the largest lie together
    x[5] = -torch.arange(40000).float().to(dtype)
    check(x, t, 32)


@pytest.mark.parametrize("low", [-math.inf, "lowest"])
@pytest.mark.parametrize("dtype", DT)
def test_masked_logits(dtype, low):
    low = torch.finfo(dtype).min if low == "lowest" else low
    x, t, g = make(8, 33000, dtype)
    keep = [0, 1, 3, 19, 20, 40, 5000, 33000]
    for r, n in enumerate(keep):
        hide = torch.ones(33000, dtype=torch.bool)
        hide[torch.randperm(33000, generator=g)[:n]] = False
        x[r, hide] = low
    lp, en, tl, ti = run(x, t, 20, 1.3)
    a, b, c, d = logprob_reference(x, 1.3, t, 20)
    assert torch.equal(ti, d)
    if low != -math.inf:                                   # scale * lowest overflows fp32: weight 0
        a = torch.where(a < -1e30, -math.inf, a)
        c = torch.where(c < -1e30, -math.inf, c)
        lp = torch.where(lp < -1e30, -math.inf, lp)
        tl = torch.where(tl < -1e30, -math.inf, tl)
    close(lp, a, torch.where(torch.isfinite(a), a.abs(), torch.zeros_like(a)).clamp_min(1.0))
    close(tl, c, torch.where(torch.isfinite(c), c.abs(), torch.zeros_like(c)).clamp_min(1.0))
    close(en, b, b.abs().clamp_min(1.0) * 2)


@pytest.mark.parametrize("dtype", DT)
def test_large_offsets_and_peaked_rows(dtype):
    x, t, _ = make(4, 20000, dtype)
    x[0] = (x[0].float() + 30000).to(dtype)
    x[1] = (x[1].float() - 30000).to(dtype)
    x[2, 11] = 400.0
    x[3] = (x[3].float() * 1e30).to(dtype)
    check(x, t, 8)


@pytest.mark.parametrize("dtype", DT)
def test_nan_and_infinity(dtype):
    x, t, _ = make(3, 20000, dtype)
    x[0, 17000] = math.nan
    x[1, 5] = math.inf
    lp, en, tl, ti = run(x, t, 4, flags=kl.KL_FLAG_RANGE)
    for r in (0, 1):
        assert torch.isnan(lp[r]).all() and torch.isnan(en[r]) and torch.isnan(tl[r]).all()
    y = x.clone()
    y[0, 17000] = -math.inf
    assert torch.equal(ti, logprob_reference(y, 1.0, t, 4)[3])
    a, b, c, _ = logprob_reference(x[2:], 1.0, t[2:], 4)
    close(lp[2:], a, a.abs().clamp_min(1))
    x, t, _ = make(1, 5, dtype)
    x[0, :4] = math.nan
    _, _, tl, ti = run(x, t, 3, flags=kl.KL_FLAG_RANGE)
    assert ti.tolist() == [[4, -1, -1]]


def test_token_ids():
    x, t, _ = make(2, 500, torch.float32)
    t[0, 0] = -1
    check(x, t, 2)
    t[1, 1], t[1, 2] = 500, -2
    lp = run(x, t, 2, flags=kl.KL_FLAG_BAD_TOKEN)[0]
    assert torch.isnan(lp[1, 1:]).all() and torch.isfinite(lp[1, 0]) and lp[0, 0] == 0


@pytest.mark.parametrize("dtype", DT)
def test_many_rows_one_workspace(dtype):
    ws = torch.zeros(1 << 24, dtype=torch.uint8, device="cuda")
    for T, V, top in ((300, 17000, 5), (1, 100000, 32), (40, 33000, 0), (300, 17000, 5)):
        x, t, _ = make(T, V, dtype, T)
        check(x, t, top, 1.0, ws=ws)


def test_no_entropy_and_no_tokens():
    x, _, _ = make(2, 30000, torch.bfloat16)
    ti = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    tl = torch.zeros((2, 3), device="cuda")
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    kl.kl_token_logprobs(2, 30000, 30000, x.cuda(), kl.KL_BF16, 0.0, None, 0, 3, None, None, tl, ti, ws)
    torch.cuda.synchronize()
    want = logprob_reference(x, 1.0, torch.zeros(2, 1), 3)
    assert torch.equal(ti.cpu(), want[3])
    close(tl.cpu(), want[2], want[2].abs().clamp_min(1))
