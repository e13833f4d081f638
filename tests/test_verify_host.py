"""Host side of the verification operators (CPU only): refusals before any launch, workspace sizes, and the
layout rule of the tree attention (csrc/kl_tree_plan.cuh, compiled for the host)."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

import paper_2606_21848_gb300 as kl
from paper_2606_21848_gb300 import builder


@pytest.fixture(scope="module", autouse=True)
def built():
    kl.build()
    kl.load()


def _shape(**kw):
    d = dict(num_seqs=2, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, num_pages=64, max_pages_per_seq=32)
    d.update(kw)
    return kl.make_shape(**d)


def _refused(status, f, *a, **kw):
    with pytest.raises(kl.KLError) as e:
        f(*a, **kw)
    assert e.value.status == status


def _tree(sh, q=16, w=16, v=16, bt=16, sl=16, cu=16, par=16, T=10, mq=8, ns=1, out=16, dt=kl.KL_FP32, ws=None):
    kl.kl_tree_attention(sh, q, w, v, bt, sl, cu, par, T, mq, ns, out, dt, ws, None, 0)


def test_tree_refusals():
    for kw in (dict(num_kv_heads=3), dict(page_size=0), dict(num_seqs=-1)):
        _refused(kl.KL_ERR_INVALID_ARG, _tree, _shape(**kw))
    for kw in (dict(T=-1), dict(mq=-1), dict(ns=-1), dict(ns=5000), dict(dt=7)):
        _refused(kl.KL_ERR_INVALID_ARG, _tree, _shape(), **kw)
    _refused(kl.KL_ERR_UNSUPPORTED, _tree, _shape(), mq=kl.KL_TREE_MAX_DRAFTS + 1)
    _refused(kl.KL_ERR_UNSUPPORTED, _tree, _shape(head_dim=64))
    assert kl.kl_tree_workspace_size(_shape(head_dim=96), 10, 8, 2) == 0
    # the shared front region, then two states of 128 rows for each run of two tiles
    assert kl.kl_tree_workspace_size(_shape(), 10, 8, 2) >= 65536 + 2 * 128 * 130 * 4


def _commit(sh, cu=16, path=16, n=16, mp=4, bt=16, sl=16, new=16, v=16):
    kl.kl_tree_commit(sh, cu, path, n, mp, bt, sl, new, v, None, 0)


def test_commit_refusals():
    _refused(kl.KL_ERR_INVALID_ARG, _commit, _shape(num_kv_heads=3))
    for kw in (dict(cu=None), dict(path=None), dict(n=None), dict(bt=None), dict(sl=None), dict(new=None),
               dict(v=None), dict(v=8), dict(mp=-1)):
        _refused(kl.KL_ERR_INVALID_ARG, _commit, _shape(), **kw)
    _commit(_shape(num_seqs=0), cu=None)              # nothing to do


def _logprobs(T=4, V=1000, stride=1000, x=16, dt=kl.KL_BF16, scale=1.0, tok=16, K=1, top=0, lp=16, en=16, tl=16,
              ti=16, ws=None):
    kl.kl_token_logprobs(T, V, stride, x, dt, scale, tok, K, top, lp, en, tl, ti, ws, None, 0)


def test_logprob_refusals():
    for kw in (dict(T=-1), dict(V=0), dict(stride=999), dict(x=None), dict(x=15), dict(dt=9), dict(K=-1),
               dict(tok=None), dict(lp=None), dict(top=-1), dict(top=1001, V=1000), dict(top=5, tl=None),
               dict(top=5, ti=None), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(x=18, dt=kl.KL_FP32)):
        _refused(kl.KL_ERR_INVALID_ARG, _logprobs, **kw)
    _refused(kl.KL_ERR_UNSUPPORTED, _logprobs, top=kl.KL_LOGPROBS_MAX_TOP + 1)
    _refused(kl.KL_ERR_WORKSPACE, _logprobs, V=100000, stride=100000)
    for bad in ("1", None, 1j):
        with pytest.raises(ctypes.ArgumentError):
            _logprobs(T=0, scale=bad)
    with pytest.raises(ctypes.ArgumentError):
        _logprobs(T=0, stride=1000.0)
    _logprobs(T=0)                                    # nothing to do
    assert kl.kl_logprobs_workspace_size(4, 1000, 5) == 0
    assert kl.kl_logprobs_workspace_size(4, 100000, 5) > 65536
    assert kl.kl_logprobs_workspace_size(4, 100000, 33) == 0


SRC = """
#include "kl_tree_plan.cuh"
extern "C" void plan(int B, int Hkv, int G, int max_q, long long tokens, int sms, int *o) {
    const kl::TreePlan p = kl::plan_tree(B, Hkv, G, max_q, tokens, sms);
    o[0] = p.hp; o[1] = p.rpb; o[2] = p.blocks; o[3] = p.ctas;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SRC)
    lib = str(d / "plan.so")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-I", builder.CSRC,
                    str(d / "plan.cpp"), "-o", lib], check=True)
    f = ctypes.CDLL(lib).plan
    f.argtypes = [ctypes.c_int] * 4 + [ctypes.c_longlong, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]

    def call(B, Hkv, G, max_q, tokens, sms=152):
        o = (ctypes.c_int * 4)()
        f(B, Hkv, G, max_q, tokens, sms, o)
        return tuple(o)
    return call


@pytest.mark.parametrize("G", [1, 2, 3, 6, 7, 8, 16, 32, 71, 128])
def test_layouts_cover_all_rows(plan, G):
    for n in (1, 2, 15, 16, 17, 33, 64, 127, 128):
        for B in (0, 1, 3, 300):
            for tokens in (16, 127, 128, 129, 5000, 131072, 1 << 29):
                hp, rpb, blocks, ctas = plan(B, 2, G, n, tokens)
                assert 1 <= hp <= G and hp * rpb <= 128
                assert blocks == -(-G // hp) * -(-n // rpb)
                assert blocks <= G * -(-n // 128)
                units = max(B, 1) * 2 * blocks
                assert ctas == min(152, max(units, (-(-tokens // 128) + 5) * units // 7))
