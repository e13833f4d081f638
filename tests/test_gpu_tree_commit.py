"""kl_tree_commit: the accepted rows bit for bit in place, everything else untouched, lengths, refusals."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def make(lens, drafts, Hkv=2, D=128, P=16, seed=0):
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // P) for n in lens]
    v = torch.randint(-2 ** 15, 2 ** 15, (sum(need), Hkv, P, D), generator=g, dtype=torch.int16)
    ids = torch.randperm(sum(need), generator=g).to(torch.int32)
    bt = torch.full((len(lens), max(need)), -1, dtype=torch.int32)
    o = 0
    for b, n in enumerate(need):
        bt[b, :n] = ids[o:o + n]
        o += n
    cu = torch.tensor([0] + torch.tensor(drafts).cumsum(0).tolist(), dtype=torch.int32)
    return v, bt, torch.tensor(lens, dtype=torch.int32), cu


def run(v, bt, lens, cu, paths, width=None, flags=0, in_place=False, max_path=None):
    width = width or max(1, max(len(p) for p in paths))
    path = torch.full((len(paths), width), 99, dtype=torch.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = torch.tensor(p, dtype=torch.int32)
    n = torch.tensor([len(p) for p in paths], dtype=torch.int32).cuda()
    pages, Hkv, P, D = v.shape
    sh = kl.make_shape(len(paths), Hkv, Hkv, D, P, pages, bt.shape[1])
    c, sl = v.cuda(), lens.cuda()
    new = sl if in_place else torch.full_like(sl, -5)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kl.kl_tree_commit(sh, cu.cuda(), path.cuda(), n, width, bt.cuda(), sl, new, c, err)
    torch.cuda.synchronize()
    assert int(err.item()) == flags
    return c.cpu(), new.cpu()


def reference(v, bt, lens, cu, paths):
    want, P = v.clone(), v.shape[2]
    new = lens.clone()
    for b, p in enumerate(paths):
        base = int(lens[b]) - int(cu[b + 1] - cu[b])
        for j, i in enumerate(p):
            s, d = base + i, base + j
            want[int(bt[b, d // P]), :, d % P] = v[int(bt[b, s // P]), :, s % P]
        new[b] = base + len(p)
    return want, new


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("P", [16, 32, 128])
@pytest.mark.parametrize("Hkv", [1, 8, 40])
@pytest.mark.parametrize("in_place", [False, True])
def test_paths(D, P, Hkv, in_place):
    lens, drafts = (300, 47, 20, 128, 9, 5), (40, 47, 3, 128, 0, 5)
    x = make(lens, drafts, Hkv, D, P, P)
    g = torch.Generator().manual_seed(Hkv)
    paths = [sorted(torch.randperm(n, generator=g)[:k].tolist())
             for n, k in zip(drafts, (7, 33, 0, 128, 0, 1))]
    got, new = run(*x, paths, in_place=in_place)
    want, lens_want = reference(*x, paths)
    assert torch.equal(got, want) and torch.equal(new, lens_want)


def test_refused_sequences_stay_as_they_are():
    x = make((100, 60, 80), (10, 8, 6))
    v, bt, lens, cu = x
    good = [[0, 3], [1, 2, 7], [5]]
    for bad, flags in (([2, 2], kl.KL_FLAG_BAD_TREE), ([3, 1], kl.KL_FLAG_BAD_TREE), ([8], kl.KL_FLAG_BAD_TREE),
                       ([-1, 2], kl.KL_FLAG_BAD_TREE), (list(range(9)), kl.KL_FLAG_BAD_TREE)):
        paths = [good[0], bad, good[2]]
        got, new = run(v, bt, lens, cu, paths, flags=flags)
        want, lens_want = reference(v, bt, lens, cu, [good[0], [], good[2]])
        lens_want[1] = -5
        assert torch.equal(got, want) and torch.equal(new, lens_want)
    short = lens.clone()
    short[1] = 7
    got, new = run(v, bt, short, cu, good, flags=kl.KL_FLAG_BAD_LENGTH)
    assert new[1] == -5
    pages = bt.clone()
    pages[1, 3] = v.shape[0]
    got, new = run(v, pages, lens, cu, good, flags=kl.KL_FLAG_BAD_PAGE)
    assert new[1] == -5 and torch.equal(got, reference(v, bt, lens, cu, [good[0], [], good[2]])[0])
