"""What the operators of a bounded cache refuse before anything is launched, and their workspaces (CPU only)."""
from __future__ import annotations

import pytest

import paper_2606_21848_gb300 as kl

INVALID, UNSUPPORTED, WORKSPACE = kl.KL_ERR_INVALID_ARG, kl.KL_ERR_UNSUPPORTED, kl.KL_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    kl.build()
    kl.load()


def shape(**kw):
    d = dict(num_seqs=2, num_q_heads=8, num_kv_heads=2, head_dim=128, page_size=16, num_pages=64, max_pages_per_seq=32)
    d.update(kw)
    return kl.make_shape(**d)


class Buffer:
    """A workspace of n bytes at an address."""

    def __init__(self, n, at=256):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


BIG = Buffer(1 << 40)


def window(sh=None, q=16, w=16, v=16, bt=16, sl=16, cu=16, total=4, max_q=2, W=100, S=4, splits=0, out=16, dt=kl.KL_BF16,
           ws=BIG):
    kl.kl_window_attention(sh or shape(), q, w, v, bt, sl, cu, total, max_q, W, S, splits, out, dt, ws, None, 0)


def weights(sh=None, q=16, w=16, v=16, bt=16, sl=16, cu=16, total=4, max_q=2, old=16, stride=512, decay=1.0, new=16,
            splits=0, out=16, dt=kl.KL_BF16, ws=BIG):
    kl.kl_attention_weights(sh or shape(), q, w, v, bt, sl, cu, total, max_q, old, stride, decay, new, splits, out, dt, ws,
                            None, 0)


def evict(sh=None, old=16, stride=512, budget=64, sinks=4, recent=16, bt=16, sl=16, nt=16, v=16, new=16, kept=16, nl=16,
          ws=BIG):
    kl.kl_evict(sh or shape(), old, stride, budget, sinks, recent, bt, sl, nt, v, new, kept, nl, ws, None, 0)


def refused(status, f, **kw):
    with pytest.raises(kl.KLError) as e:
        f(**kw)
    assert e.value.status == status, kw


@pytest.mark.parametrize("f", [window, weights])
def test_attention_arguments(f):
    for bad in (dict(num_kv_heads=3), dict(page_size=0), dict(num_pages=0), dict(num_seqs=-1), dict(max_pages_per_seq=0)):
        refused(INVALID, f, sh=shape(**bad))
    for kw in (dict(total=-1), dict(max_q=-1), dict(splits=-1), dict(splits=1 << 20), dict(dt=7)):
        refused(INVALID, f, **kw)


def test_their_own_arguments():
    for kw in (dict(W=0), dict(W=-1), dict(S=-1)):
        refused(INVALID, window, **kw)
    for kw in (dict(stride=0), dict(decay=-0.5), dict(decay=float("nan")), dict(decay=float("inf"))):
        refused(INVALID, weights, **kw)
    refused(UNSUPPORTED, weights, max_q=kl.KL_WEIGHTS_MAX_ROWS + 1)


def test_unsupported_shapes():
    for f in (window, weights):
        for bad in (dict(head_dim=96), dict(head_dim=64), dict(page_size=24), dict(num_q_heads=512)):
            refused(UNSUPPORTED, f, sh=shape(**bad))


def test_window_workspace():
    def size(sh=None, total=4, max_q=2, W=100, S=4, splits=0):
        return kl.kl_window_workspace_size(sh or shape(), total, max_q, W, S, splits)

    assert size() > 0
    for kw in (dict(sh=shape(num_kv_heads=3)), dict(total=-1), dict(max_q=-1), dict(W=0), dict(W=-5), dict(S=-1),
               dict(splits=-1)):
        assert size(**kw) == 0, kw
    # the window bounds the states, not the table; sizes beyond the longest sequence are that sequence's
    long = shape(max_pages_per_seq=1 << 16)
    assert size(long, W=1 << 30) == size(long, W=1 << 20)
    assert size(long, S=(1 << 31) - 1) == size(long, S=1 << 20)


def test_weights_workspace():
    def size(sh=None, total=4, max_q=2, stride=512, splits=0):
        return kl.kl_weights_workspace_size(sh or shape(), total, max_q, stride, splits)

    # at least the scores: 2 sequences, 8 heads, 2 rows, 512 tokens
    assert size() >= 2 * 8 * 2 * 512 * 4
    for kw in (dict(sh=shape(num_kv_heads=3)), dict(total=-1), dict(max_q=-1), dict(stride=0), dict(splits=-1),
               dict(max_q=kl.KL_WEIGHTS_MAX_ROWS + 1)):
        assert size(**kw) == 0, kw
    assert size(shape(num_seqs=64, max_pages_per_seq=1 << 13), max_q=128, stride=1 << 17) > 1 << 32


def test_evict_arguments():
    for kw in (dict(stride=0), dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=60, recent=5),
               dict(sinks=(1 << 31) - 1, recent=1), dict(sh=shape(num_kv_heads=3)), dict(old=None), dict(bt=None),
               dict(sl=None), dict(nt=None), dict(v=None), dict(v=8), dict(new=None), dict(kept=None), dict(nl=None),
               dict(old=2), dict(new=2)):
        refused(INVALID, evict, **kw)
    refused(UNSUPPORTED, evict, sh=shape(head_dim=96))
    long = shape(max_pages_per_seq=1 << 16)
    refused(UNSUPPORTED, evict, sh=long, stride=kl.KL_EVICT_MAX_TOKENS + 1)
    for ws in (None, Buffer(0), Buffer(kl.kl_evict_workspace_size(shape(), 512, 64) - 1), Buffer(1 << 30, 128)):
        refused(WORKSPACE, evict, ws=ws)
    assert evict(sh=shape(num_seqs=0)) is None            # nothing to do
    assert kl.kl_evict_workspace_size(shape(), 512, 0) == 0


def test_weights_of_more_sequences_than_a_grid_has():
    for bad in (dict(num_seqs=65536), dict(num_q_heads=65536, num_kv_heads=65536)):
        refused(UNSUPPORTED, weights, sh=shape(**bad))
        assert kl.kl_weights_workspace_size(shape(**bad), 4, 2, 512, 0) == 0
