"""The barriers of the tree attention's pipeline (csrc/kl_tree_tc.cu), on the CPU: every wait by parity is for a
phase that it cannot miss.

A wait for phase n of a barrier passes while the barrier is in phase n + 1. Before phase n - 1 is complete it
passes at once, and after phase n + 1 it blocks. So of what the waiter has seen before it waits phase n - 1 has
to follow, and the completion of phase n + 1 has to follow from the wait itself, whatever the warps' speeds. The
steps of a segment and what each waits for are written down here as a graph; the sizes are the kernel's."""
from __future__ import annotations

import os
import re
import subprocess

import pytest

from paper_2606_21848_gb300 import builder

NAMES = ("kTreeGroups", "kTreeSub", "kTreeSubFp32", "kTreeFold", "kTreeTurns")


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    d = tmp_path_factory.mktemp("sizes")
    (d / "sizes.cpp").write_text('#include <cstdio>\n#include "kl_tree_plan.cuh"\nint main() { std::printf("' +
                                 " ".join(f"{n}=%d" for n in NAMES) + '", ' + ", ".join("kl::" + n for n in NAMES) +
                                 "); }\n")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-I", builder.CSRC, str(d / "sizes.cpp"), "-o",
                    str(d / "sizes")], check=True)
    out = subprocess.run([str(d / "sizes")], check=True, capture_output=True, text=True).stdout
    return {k: int(v) for k, v in re.findall(r"(\w+)=(\d+)", out)}


class Graph:
    """Steps, what each follows, and waits (step, barrier, phase). A step is done in order behind `after` (the
    same warps' earlier steps) and behind the phases that it waits for, in the order given."""

    def __init__(self):
        self.before, self.completes, self.waits = {}, {}, []

    def step(self, name, after=(), waits=(), completes=None):
        """waits: [(barrier, phase)]; completes: the (barrier, phase) that the step completes."""
        known = [a for a in after if a in self.before]
        for barrier, phase in waits:
            self.waits.append((name, barrier, phase, tuple(known)))
            known.append((barrier, phase))
        self.before[name] = known
        if completes:
            self.completes[completes] = name

    def resolve(self):
        for name, known in self.before.items():
            self.before[name] = {k if k in self.before else self.completes[k] for k in known}

    def ancestors(self, names):
        seen, todo = set(), list(names)
        while todo:
            n = todo.pop()
            if n not in seen:
                seen.add(n)
                todo += self.before[n]
        return seen

    def faults(self):
        self.resolve()
        bad = []
        for name, barrier, phase, known in self.waits:
            known = [k if k in self.before else self.completes[k] for k in known]
            earlier = self.completes.get((barrier, phase - 1))
            if earlier is not None and earlier not in self.ancestors(known):
                bad.append((name, barrier, phase, "early"))
            later = self.completes.get((barrier, phase + 1))
            if later is not None and name not in self.ancestors([later]):
                bad.append((name, barrier, phase, "late"))
        return bad


def fp32(n, groups, sub, fold, turns):
    """A segment of n half tiles with fp32 outputs. S: scores, T: the reference is announced, P: the weights are
    there, V: the output products are done, F: O moves to the sum before half tile u."""
    g = Graph()
    for u in range(n):
        g.step(("S", u), [("S", u - 1)], [(("s_free", (u - sub) % 4), (u - sub) // 4)] if u >= sub else [],
               (("s_full", u % 4), u // 4))
        turn = [(("turn", (u - 1) % turns), (u - 1) // turns)] if u else []
        g.step(("T", u), [("P", u - groups)], [(("s_full", u % 4), u // 4)] + turn, (("turn", u % turns), u // turns))
        g.step(("P", u), [("T", u)], [], (("p_full", u % 4), u // 4))
        waits = [(("p_full", u % 4), u // 4)]
        if u and u % fold == 0:
            waits.append((("o_free", 0), u // fold - 1))
            g.step(("F", u), [("F", u - fold)], [(("s_free", (u - 1) % 4), (u - 1) // 4),
                                                 (("turn", (u - 1) % turns), (u - 1) // turns)],
                   (("o_free", 0), u // fold - 1))
        g.step(("V", u), [("V", u - 1)], waits, (("s_free", u % 4), u // 4))
    return g


def test_fp32_outputs(sizes):
    for n in range(1, 24):
        assert fp32(n, sizes["kTreeGroups"], sizes["kTreeSubFp32"], sizes["kTreeFold"], sizes["kTreeTurns"]).faults() == []


def test_a_barrier_per_group_would_be_missed(sizes):
    """The graph shows the fault of announcing on a barrier per group: the moves of O may come too late."""
    bad = fp32(12, sizes["kTreeGroups"], sizes["kTreeSubFp32"], sizes["kTreeFold"], sizes["kTreeGroups"]).faults()
    assert bad and all(step[0] == "F" and why == "late" for step, _, _, why in bad)


def bf16(n, groups, sub):
    """A segment of n half tiles with bf16 outputs: S scores, R behind a wait that a reference which moves adds, P
    weights, V output products, E the epilogues. Each group has its own reference and O."""
    g = Graph()
    for u in range(n):
        g.step(("S", u), [("S", u - 1)], [(("s_free", (u - sub) % 4), (u - sub) // 4)] if u >= sub else [],
               (("s_full", u % 4), u // 4))
        seen = [(("s_full", u % 4), u // 4)]
        g.step(("R", u), [("P", u - groups)],
               seen + ([(("s_free", (u - groups) % 4), (u - groups) // 4)] if u >= groups else []))
        g.step(("P", u), [("P", u - groups)], seen, (("p_full", u % 4), u // 4))
        g.step(("V", u), [("V", u - 1)], [(("p_full", u % 4), u // 4)], (("s_free", u % 4), u // 4))
    last = n - 1
    for grp in range(groups):
        mine = [u for u in range(n) if u % groups == grp]
        g.step(("E", grp), [("P", mine[-1])] if mine else [],
               [(("s_free", u % 4), u // 4) for u in range(last, max(last - 3, -1), -1)])
    return g


def test_bf16_outputs(sizes):
    for n in range(1, 24):
        # (R is on P's way where it is waited for, so what follows from P follows from it)
        faults = bf16(n, sizes["kTreeGroups"], sizes["kTreeSub"]).faults()
        assert [f for f in faults if f[0][0] != "R" or f[3] != "late"] == []


def test_all_scores_and_output_products_are_waited_for(sizes):
    """What ends a segment sees every completion on the barriers of scores and weights, which are then set up anew."""
    for n in range(1, 24):
        g = bf16(n, sizes["kTreeGroups"], sizes["kTreeSub"])
        g.resolve()
        waited = g.ancestors([("E", e) for e in range(sizes["kTreeGroups"])])
        assert {("V", u) for u in range(n)} | {("S", u) for u in range(n)} <= waited
