"""Refusals of kvb_accept (no GPU)."""
import ctypes

import pytest

from paper_2605_19049_amd import kvb

A = 0x1000   # a fake, well-aligned "device address"
GOOD = dict(B=2, T=4, V=1000, dtype=kvb.F32)


def _accept(vo, **kw):
    d = dict(n_drafts=None, parent=None, tokens=A, target=A, draft=A, u=A, s=A, path=A, accepted=A, token=A, work=A)
    d.update(kw)
    return kvb.kvb_accept(vo, *d.values(), stream=0, check=False)


def test_struct_layout_matches_header():
    assert ctypes.sizeof(kvb.KvbVocab) == 24 and kvb.KvbVocab.stride.offset == 16


@pytest.mark.parametrize("bad, code", [(dict(B=-1), kvb.EINVAL), (dict(B=(1 << 20) + 1), kvb.EINVAL), (dict(T=0), kvb.EINVAL), (dict(T=9), kvb.EINVAL),
                                       (dict(V=0), kvb.EINVAL), (dict(V=(1 << 24) + 1), kvb.EINVAL), (dict(dtype=3), kvb.EUNSUPPORTED),
                                       (dict(stride=999), kvb.EINVAL), (dict(stride=-1000), kvb.EINVAL), (dict(stride=1 << 40), kvb.EINVAL)])
def test_bad_sizes_are_rejected(bad, code):
    vo = kvb.vocab(**{**GOOD, **bad})
    assert _accept(vo) == code
    assert kvb.lib().kvb_accept_work(ctypes.byref(vo)) == code


@pytest.mark.parametrize("bad", [dict(tokens=None), dict(target=None), dict(u=None), dict(s=None), dict(path=None), dict(accepted=None), dict(token=None),
                                 dict(work=None), dict(target=A + 2), dict(draft=A + 1), dict(parent=A + 2), dict(n_drafts=A + 1), dict(u=A + 2),
                                 dict(work=A + 4)])
def test_bad_pointers_are_rejected(bad):
    assert _accept(kvb.vocab(**GOOD), **bad) == kvb.EINVAL


def test_nothing_to_do():
    assert _accept(kvb.vocab(**{**GOOD, "B": 0}), tokens=None, target=None) == kvb.OK
    with pytest.raises(kvb.KvbError):
        kvb.accept_work(kvb.vocab(**{**GOOD, "T": 9}))
