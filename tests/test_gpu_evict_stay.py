"""Rows that an eviction in place leaves where they are: they are not copied onto themselves, and what does move is right
wherever the first row that goes lies."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import workspace
from tests.test_gpu_evict import case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    kl.build()
    kl.load()


def falling_from(c, first):
    """Weights of which token `first` has the least, and every later one the more the earlier it lies."""
    E = c["w"].shape[2]
    t = torch.arange(E)
    c["w"][:] = torch.where(t < first, 2.0 * E, torch.where(t == first, 0.25, (E - t).float()))
    return c


@pytest.mark.parametrize("first", [0, 1, 31, 32, 63, 64, 65, 500, 991])
@pytest.mark.parametrize("Hkv,D", [(1, 128), (2, 64), (24, 64)])
def test_the_first_row_that_goes(first, Hkv, D):
    """Two to 48 value heads: each form of the move; one row goes, or some more."""
    check(falling_from(case((1000, 700), Hkv, D, 16), first), 999, 0, 0)
    check(falling_from(case((1000, 700), Hkv, D, 16), first), 990, 0, 0, in_place=True)


@pytest.mark.parametrize("first", [4095, 20480, 39990])
def test_the_first_row_that_goes_in_a_cluster(first):
    check(falling_from(case((40000,), 1, 64, 16), first), 39999, 0, 0)


def test_sequences_within_their_budget():
    for Hkv in (2, 40):
        check(case((500, 64, 63, 0, 700), Hkv), 700, 4, 16, in_place=True)
        c = case((500, 64, 63, 0, 700), Hkv, spare=1)
        c["other"][:, :3] = c["table"][:, :3]          # some pages stay, others are new
        check(c, 700, 4, 16)


@pytest.mark.parametrize("B,Hkv,L", [(64, 8, 4096), (1, 8, 200000)])
def test_nothing_is_copied_onto_itself(B, Hkv, L):
    """A batch within its budget in place takes the selection's time alone: less than half of what its copy to other pages
    takes (about a fifth; with every row rewritten the two take the same)."""
    P = 64
    pages = -(-L // P)
    table = torch.arange(B * pages, dtype=torch.int32, device="cuda").view(B, pages)
    other = table + B * pages
    v = torch.zeros(2 * B * pages, Hkv, P, 128, dtype=torch.bfloat16, device="cuda")
    w, lens = torch.rand(B, Hkv, L, device="cuda"), torch.full((B,), L, dtype=torch.int32, device="cuda")
    new, new_lens = torch.zeros_like(w), torch.zeros_like(lens)
    kept = torch.zeros(B, Hkv, L, dtype=torch.int32, device="cuda")
    sh = kl.make_shape(B, Hkv, Hkv, 128, P, 2 * B * pages, pages)
    ws = workspace(kl.kl_evict_workspace_size(sh, L, L))

    def us(to):
        best = 1e9
        for _ in range(8):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(4):
                kl.kl_evict(sh, w, L, L, 4, 64, table, lens, to, v, new, kept, new_lens, ws)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b) / 4 * 1e3)
        return best

    stays, moves = us(table), us(other)
    print(f"in place {stays:.1f} us, to other pages {moves:.1f} us")
    assert stays < 0.5 * moves
