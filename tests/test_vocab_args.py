"""Refusals of the vocabulary losses: found on the host, before any CUDA call, so they run without a GPU."""
import ctypes as C

import pytest

import paper_1805_10111_b200 as dq
from paper_1805_10111_b200 import build as dq_build

P = 1 << 20                                  # a pointer-like number, 256-byte aligned; never followed


@pytest.fixture(scope="module")
def L():
    dq_build.build()
    return dq.lib()


def _v(**kw):
    f = dict(format=dq.DQ_DENSE_F32, k=0, n=8, d=16, V=32, h=P, ld_h=16, w=P, ld_w=16, workspace=P, workspace_bytes=1 << 40)
    f.update(kw)
    return dq.dq_vocab(*[f[k] for k, _ in dq.dq_vocab._fields_])


def _calls(L, v, labels=P, loss=P, lse=P, weight=None, gh=P, ld_gh=16, gw=P, ld_gw=16, idx=P, t=P, temp=1.0):
    """Status of all four entry points: cross-entropy loss and gradient (k as given), distillation loss and gradient."""
    r = C.byref(v)
    return (L.dq_xent_loss(r, labels, loss, lse, None), L.dq_xent_grad(r, labels, weight, loss, lse, gh, ld_gh, gw, ld_gw, None),
            L.dq_distill_loss(r, idx, t, None, temp, loss, lse, None),
            L.dq_distill_grad(r, idx, t, None, temp, weight, loss, lse, gh, ld_gh, gw, ld_gw, None))


@pytest.mark.parametrize("bad", [dict(format=dq.DQ_CSR_F32), dict(format=7), dict(n=-1), dict(n=(1 << 24) + 1), dict(d=0), dict(d=(1 << 16) + 1),
                                 dict(V=0), dict(V=(1 << 28) + 1), dict(n=1 << 24, V=1 << 24), dict(ld_h=15), dict(ld_w=15), dict(ld_w=-1), dict(ld_h=1 << 40), dict(w=None),
                                 dict(h=None), dict(workspace=None), dict(workspace=P + 16), dict(h=P + 2), dict(w=P + 1)])
def test_bad_descriptors(L, bad):
    k = {k: v for k, v in bad.items()}
    assert _calls(L, _v(**k))[:2] == (dq.DQ_ERR_ARG,) * 2
    assert _calls(L, _v(**dict(k, k=4)))[2:] == (dq.DQ_ERR_ARG,) * 2
    if set(bad) & {"format", "n", "d", "V"} or bad.get("ld_w", 16) < 16 or "ld_h" in bad:
        assert L.dq_vocab_workspace_bytes(C.byref(_v(**k)), 1) == -1


def test_bad_arguments(L):
    assert _calls(L, _v(), labels=None)[:2] == (dq.DQ_ERR_ARG,) * 2
    assert _calls(L, _v(), loss=None)[:2] == (dq.DQ_ERR_ARG,) * 2
    assert _calls(L, _v(k=3), idx=None)[2:] == (dq.DQ_ERR_ARG,) * 2
    assert _calls(L, _v(k=3), t=None)[2:] == (dq.DQ_ERR_ARG,) * 2
    assert _calls(L, _v(), labels=P + 2)[:2] == (dq.DQ_ERR_ARG,) * 2
    for temp in (0.0, -1.0, float("nan"), float("inf"), 1e-39):
        assert _calls(L, _v(k=3), temp=temp)[2:] == (dq.DQ_ERR_ARG,) * 2
    for kw in (dict(gh=None), dict(gw=None), dict(ld_gh=15), dict(ld_gw=15), dict(ld_gh=1 << 40), dict(ld_gw=1 << 40), dict(gh=P + 2), dict(gw=P + 2), dict(weight=P + 1)):
        assert _calls(L, _v(), **kw)[1] == dq.DQ_ERR_ARG
        assert _calls(L, _v(k=3), **kw)[3] == dq.DQ_ERR_ARG


def test_number_of_entries_decides_the_loss(L):
    assert _calls(L, _v(k=3))[:2] == (dq.DQ_ERR_ARG,) * 2                         # entries given to a call that takes labels
    assert _calls(L, _v(k=0))[2:] == (dq.DQ_ERR_ARG,) * 2
    for k in (-1, dq.DQ_VOCAB_MAX_TOP + 1):
        assert _calls(L, _v(k=k)) == (dq.DQ_ERR_ARG,) * 4


def test_null_descriptor(L):
    assert L.dq_xent_loss(None, P, P, P, None) == dq.DQ_ERR_ARG
    assert L.dq_xent_grad(None, P, None, P, P, P, 16, P, 16, None) == dq.DQ_ERR_ARG
    assert L.dq_distill_loss(None, P, P, None, 1.0, P, P, None) == dq.DQ_ERR_ARG
    assert L.dq_distill_grad(None, P, P, None, 1.0, None, P, P, P, 16, P, 16, None) == dq.DQ_ERR_ARG
    assert L.dq_vocab_workspace_bytes(None, 0) == -1
    s = C.c_int(0)
    assert L.dq_vocab_status(None, C.byref(s), None) == dq.DQ_ERR_ARG
    assert L.dq_vocab_status(C.byref(_v(workspace=None)), C.byref(s), None) == dq.DQ_ERR_ARG


def test_holder_refuses_other_types_and_shapes():
    torch = pytest.importorskip("torch")
    h, w = torch.zeros(4, 8), torch.zeros(9, 8)
    for a, b in ((h, w), (h.half(), w.half()), (h, w.bfloat16()), (h.double(), w.double()), (h[0], w), (h, w[:, :7])):
        with pytest.raises(dq.DqError):
            dq.Vocab(a, b, workspace=torch.zeros(1 << 20, dtype=torch.uint8))
