"""Refusals of kvb_scan and the sizes of its workspace (no GPU)."""
import ctypes

import pytest
import torch

from paper_2605_19049_amd import kvb

A = 0x1000   # a fake, well-aligned "device address"
GOOD = dict(B=2, Hk=2, Hv=4, dk=128, dv=128, cap=1, in_dtype=kvb.BF16)


def _seqs(**kw):
    d = dict(start=A, n_tokens=100, n_slots=4, slot=A)
    d.update({x: kw.pop(x) for x in list(kw) if x in d})
    sq = kvb.seqs(**d)
    for x, y in kw.items():
        setattr(sq, x, y)
    return sq


def _scan(sh, sq, **kw):
    d = dict(q=A, k=A, v=A, g=A, beta=A, state0=A, state1=A, out=A, work=A)
    d.update(kw)
    return kvb.kvb_scan(sh, sq, *d.values(), stream=0, check=False)


def test_struct_layout_matches_header():
    assert ctypes.sizeof(kvb.KvbSeqs) == 48
    assert kvb.KvbSeqs.q_stride.offset == 16 and kvb.KvbSeqs.n_tokens.offset == 40 and kvb.KvbSeqs.n_slots.offset == 44


@pytest.mark.parametrize("bad, code", [
    (dict(B=-1), kvb.EINVAL), (dict(Hk=0), kvb.EINVAL), (dict(Hk=3), kvb.EINVAL), (dict(dv=0), kvb.EINVAL),
    (dict(dk=96, dv=96), kvb.EUNSUPPORTED), (dict(dk=128, dv=64), kvb.EUNSUPPORTED), (dict(in_dtype=3), kvb.EUNSUPPORTED),
    (dict(out_dtype=kvb.F16), kvb.EUNSUPPORTED), (dict(in_dtype=kvb.F32, out_dtype=kvb.BF16), kvb.EUNSUPPORTED),
    (dict(B=1 << 30), kvb.EINVAL), (dict(Hk=1 << 20, Hv=1 << 20, B=1 << 9), kvb.EINVAL)])
def test_bad_shapes_are_rejected(bad, code):
    sh = kvb.shape(**{**GOOD, **bad})
    assert _scan(sh, _seqs()) == code
    assert kvb.lib().kvb_scan_work(ctypes.byref(sh), ctypes.byref(_seqs())) == code


@pytest.mark.parametrize("bad", [dict(n_tokens=-1), dict(n_slots=-1), dict(q_stride=255), dict(k_stride=260), dict(v_stride=8), dict(v_stride=-512),
                                 dict(q_stride=1 << 62), dict(start=None), dict(start=A + 2), dict(slot=A + 1)])
def test_bad_sequences_are_rejected(bad):
    assert _scan(kvb.shape(**GOOD), _seqs(**bad)) == kvb.EINVAL


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=A + 8), dict(v=None), dict(g=None), dict(beta=A + 2), dict(state0=A + 4), dict(state1=A + 8),
                                 dict(out=None), dict(out=A + 8), dict(work=None), dict(work=A + 8)])
def test_bad_pointers_are_rejected(bad):
    assert _scan(kvb.shape(**GOOD), _seqs(), **bad) == kvb.EINVAL


def test_nothing_to_do():
    assert _scan(kvb.shape(**{**GOOD, "B": 0}), _seqs()) == kvb.OK
    assert _scan(kvb.shape(**{**GOOD, "B": 0}), _seqs(n_tokens=0), q=None, out=None, work=None) == kvb.OK
    with pytest.raises(kvb.KvbError):
        kvb.scan_work(kvb.shape(**{**GOOD, "dk": 96}), _seqs())


def test_workspace_grows_with_what_it_depends_on():
    def size(B, Hv, n):
        return kvb.scan_work(kvb.shape(**{**GOOD, "B": B, "Hv": Hv}), _seqs(n_tokens=n))
    assert size(1, 4, 64) < size(2, 4, 64) < size(2, 8, 64) < size(2, 8, 6400)
    assert size(1, 32, 1 << 20) > 1 << 31   # (64-bit sizes)


def test_strides_of_tensors():
    x = torch.zeros(10, 7 * 64)
    q = x[:, :128].view(10, 2, 64)
    assert kvb.seqs(A, 10, 1, q=q).q_stride == 7 * 64
    assert kvb.seqs(A, 1, 1, q=q[:1]).q_stride == 0
    assert kvb.seqs(A, 10, 1, v=torch.zeros(10, 2, 64)).v_stride == 128
    for bad in (q.transpose(0, 1).contiguous().transpose(0, 1), q[:, :, ::2], torch.zeros(1, 2, 64).expand(10, 2, 64)):
        with pytest.raises(ValueError):
            kvb.seqs(A, 10, 1, q=bad)


def _backward(sh, sq, **kw):
    d = dict(q=A, k=A, v=A, g=A, beta=A, state0=A, dout=A, dstate1=A, dq=A, dk=A, dv=A, dg=A, dbeta=A, dstate0=A, work=A)
    d.update(kw)
    return kvb.kvb_scan_backward(sh, sq, *d.values(), stream=0, check=False)


@pytest.mark.parametrize("bad", [dict(q=A + 8), dict(dout=None), dict(dout=A + 8), dict(dq=None), dict(dk=A + 2), dict(dv=None), dict(dg=None), dict(dbeta=A + 2),
                                 dict(dstate1=A + 8), dict(dstate0=A + 4), dict(work=None), dict(beta=None)])
def test_bad_pointers_of_the_backward_pass(bad):
    assert _backward(kvb.shape(**GOOD), _seqs(), **bad) == kvb.EINVAL


def test_backward_pass_refuses_what_the_forward_pass_does():
    assert _backward(kvb.shape(**{**GOOD, "dk": 96, "dv": 96}), _seqs()) == kvb.EUNSUPPORTED
    assert _backward(kvb.shape(**GOOD), _seqs(q_stride=255)) == kvb.EINVAL
    assert _backward(kvb.shape(**{**GOOD, "B": 0}), _seqs()) == kvb.OK
    assert kvb.scan_backward_work(kvb.shape(**GOOD), _seqs()) > kvb.scan_work(kvb.shape(**GOOD), _seqs())
