"""How blocks of consecutive positions are cut into runs (csrc/kl_window.cuh), compiled for the host: every cut covers
its line, and no block has more runs than the CTA that merges them has room for."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

from paper_2606_21848_gb300 import builder

MOST = 256                # states that one CTA merges
SRC = """
#include <stdint.h>
#define __host__
#define __device__
#include "kl_window.cuh"
extern "C" void runs(long long units, long long tokens, int splits, long long slots, int most, int *out) {
    const kl::CausalRuns r = kl::plan_runs(units, tokens, splits, slots, most);
    out[0] = r.splits; out[1] = r.chunk; out[2] = r.spc; out[3] = r.whole;
}
extern "C" int most_runs() { return kl::kCausalMostRuns; }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SRC)
    so = str(d / "plan.so")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-I", builder.CSRC,
                    str(d / "plan.cpp"), "-o", so], check=True)
    return ctypes.CDLL(so)


def runs(lib, units, tokens, splits, slots, most=MOST):
    out = (ctypes.c_int * 4)()
    L = ctypes.c_longlong
    lib.runs(L(units), L(tokens), splits, L(slots), most, out)
    return tuple(out)


def test_the_bound_is_the_merge_s(lib):
    assert lib.most_runs() == MOST


@pytest.mark.parametrize("slots", [1, 132, 152, 304])
@pytest.mark.parametrize("tokens", [1, 128, 129, 2000, 8192, 8193, 65536, 131072, (1 << 21) + 1, 4000000, (1 << 31) - 128])
def test_runs_cover_the_line_and_fit_the_merge(lib, slots, tokens):
    for units in (1, 2, 3, 7, 8, 64, 151, 152, 153, 200, 303, 304, 305, 608, 1000, 16384, 1 << 20):
        for splits in (0, 1, 2, 3, 7, 64, 152, 255, 256, 257, 384, 400, 426, 427, 512, 608, 1000, 1024):
            n, chunk, spc, whole = runs(lib, units, tokens, splits, slots)
            cut = -(-n // spc)
            assert 1 <= cut <= MOST, (units, splits, n)
            assert chunk % 128 == 0 and n * chunk >= tokens > (n - 1) * chunk, (units, splits, n, chunk)
            assert 0 <= whole <= units and (n > 1 or whole == units), (units, splits, n, whole)
            if splits:
                assert cut <= splits


def test_the_caller_s_number_of_runs(lib):
    """One unit of 65536 tokens: as many runs as asked for, up to the bound."""
    for splits, want in ((1, 1), (100, 86), (128, 128), (256, 256), (400, 256), (512, 256), (1024, 256)):
        n = runs(lib, 1, 65536, splits, 152)[0]
        assert n == want, (splits, n)
