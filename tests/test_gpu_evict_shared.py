"""Few value heads in place, whose CTAs wait for each other's reads, while another stream keeps the memory and the SMs
busy: every row that stays arrives, time after time."""
from __future__ import annotations

import pytest
import torch

import paper_2606_21848_gb300 as kl
from tests._bounded import workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L,Hkv,D,budget,kind", [(40000, 1, 128, 39000, "random"), (40000, 2, 64, 20000, "random"),
                                                 (9000, 8, 128, 8990, "random"), (60000, 1, 128, 30000, "halves"),
                                                 (30000, 4, 128, 15000, "every other")])
def test_rows_arrive_beside_other_work(L, Hkv, D, budget, kind):
    kl.build()
    kl.load()
    gen = torch.Generator(device="cuda").manual_seed(L)
    P, pages = 16, -(-L // 16)
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)[None].contiguous()
    rows = torch.randint(-32768, 32767, (pages, Hkv, P, D), generator=gen, device="cuda").to(torch.int16)
    t = torch.arange(L, device="cuda")
    w = {"random": torch.rand(1, Hkv, L, generator=gen, device="cuda"),
         "halves": (t >= L // 2).float().expand(1, Hkv, L).contiguous(),
         "every other": (t % 2).float().expand(1, Hkv, L).contiguous()}[kind]
    sh = kl.make_shape(1, Hkv, Hkv, D, P, pages, pages)
    ws, err = workspace(kl.kl_evict_workspace_size(sh, L, budget)), torch.zeros(1, dtype=torch.int32, device="cuda")
    order = torch.argsort(w[0], dim=-1, descending=True, stable=True)[:, :budget]
    want_ids = torch.sort(order, -1).values                      # [Hkv][budget]
    h, j = torch.arange(Hkv, device="cuda")[:, None], torch.arange(budget, device="cuda")
    want = rows[table[0].long()[want_ids // P], h, want_ids % P]
    kept, new = torch.zeros(1, Hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros_like(w)
    lens, new_lens = torch.tensor([L], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    other, a, b = torch.cuda.Stream(), torch.zeros(1 << 26, device="cuda"), torch.zeros(1 << 26, device="cuda")
    torch.cuda.synchronize()
    for i in range(20):
        v = rows.clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            for _ in range(3):
                b.copy_(a)
        kl.kl_evict(sh, w, L, budget, 0, 0, table, lens, table, v, new, kept, new_lens, ws, err)
        torch.cuda.synchronize()
        assert int(err) == 0 and torch.equal(kept[0].long(), want_ids)
        assert torch.equal(v[table[0].long()[j // P][None], h, j % P], want), i
