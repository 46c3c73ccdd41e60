"""What bind refuses: its calls go to the library without a further look at their arguments' types."""
import ctypes

import pytest

from paper_2605_19049_amd import kvb

A = 0x1000   # a fake, well-aligned address
SH, ST = kvb.shape(1, 2, 4, 64, 64, 8, kvb.BF16), kvb.store(A, A, A, A, A, A, 1)
TA, SQ = kvb.taps(A, A_log=A, dt_bias=A), kvb.seqs(A, 1, 1)
RO, VO, LI = kvb.rows(1, 1, 64, kvb.BF16), kvb.vocab(1, 1, 8, kvb.F32), kvb.KvbList(A, A, A, A, 1, 1)

# each call's structs, scalars and pointers in order: a struct, a number, or A
CALLS = {
    "kvb_decode": [SH, ST] + [A] * 8, "kvb_decode_flush": [SH, ST] + [A] * 7 + [1, A], "kvb_flush": [SH, ST, A, A, 1, A], "kvb_verify": [SH, ST, A, 2] + [A] * 7,
    "kvb_verify_tree": [SH, ST, A, 2] + [A] * 8, "kvb_compact": [SH, ST, A, 2] + [A] * 3, "kvb_direct": [SH, ST, A, A, 2] + [A] * 7,
    "kvb_scan": [SH, SQ] + [A] * 10, "kvb_scan_backward": [SH, SQ] + [A] * 16, "kvb_accept": [VO] + [A] * 12,
    "kvb_conv": [SH, TA, SQ] + [A] * 11, "kvb_conv_decode": [SH, TA, A, 2] + [A] * 11, "kvb_conv_verify": [SH, TA, A, 2, 2] + [A] * 11,
    "kvb_conv_commit": [SH, TA, A, 2, 2] + [A] * 6, "kvb_conv_backward": [SH, TA, SQ] + [A] * 20, "kvb_norm": [RO] + [A] * 7, "kvb_norm_backward": [RO] + [A] * 11,
    "kvb_grad_norm": [LI] + [A] * 3, "kvb_clip": [LI, LI, A, 1.0, A]}
OPTIONAL = {("kvb_clip", 1)}   # `to`


def test_every_call_is_here():
    rest = {n for n in kvb.EXPORTS if n.endswith("_work") or "timer" in n} | {"kvb_strerror", "kvb_version"}
    assert set(CALLS) == set(kvb.EXPORTS) - rest


@pytest.mark.parametrize("name", CALLS)
def test_arguments_of_another_kind(name):
    args = CALLS[name]
    kvb.bind(name, *args)
    for i, a in enumerate(args):
        def with_(x):
            return kvb.bind(name, *args[:i], x, *args[i + 1:])
        if isinstance(a, ctypes.Structure):
            wrong = [kvb.KvbStore() if isinstance(a, kvb.KvbShape) else kvb.KvbShape(), A, 1.5]
            if (name, i) in OPTIONAL:
                with_(None)
            else:
                wrong.append(None)
        elif isinstance(a, float):
            with_(3)
            wrong = [None, kvb.KvbShape(), "1"]
        elif a is not A:
            wrong = [None, 1.5, kvb.KvbShape(), "1"]
        else:
            with_(None)
            wrong = [kvb.KvbShape(), 1.5]
        for x in wrong:
            with pytest.raises(TypeError):
                with_(x)


def test_a_call_of_another_length():
    for name, args in CALLS.items():
        for other in (args[:-1], args + [A]):
            with pytest.raises(AssertionError):
                kvb.bind(name, *other)


def test_a_bound_call_passes_numbers_where_the_library_has_them():
    """An integer and a float in the middle of pointers: the library refuses what they say (before any HIP call)"""
    with pytest.raises(kvb.KvbError, match="kvb_clip"):
        kvb.bind("kvb_clip", LI, None, A, -1.0, 0)()
    with pytest.raises(kvb.KvbError, match="kvb_clip"):
        kvb.bind("kvb_clip", LI, None, A, -1, 0)()
    kvb.bind("kvb_clip", kvb.KvbList(None, None, None, None, 0, 0), None, A, 1.0, 0)()   # nothing to cut
    for n_slots, T in ((-1, 2), (2, 0), (2, kvb.MAX_DRAFTS + 1)):
        with pytest.raises(kvb.KvbError, match="kvb_conv_verify"):
            kvb.bind("kvb_conv_verify", SH, TA, A, n_slots, T, None, *[A] * 10)()


AROUND = [n for n in CALLS if n.startswith(("kvb_conv", "kvb_norm")) or n in ("kvb_grad_norm", "kvb_clip")]


@pytest.mark.parametrize("name", AROUND)
def test_a_struct_is_no_address_in_a_plain_call_either(name):
    """(sizes that the library refuses: nothing is launched)"""
    args = list(CALLS[name][:-1])
    bad = {kvb.KvbShape: kvb.shape(-1, 2, 4, 64, 64, 8, kvb.BF16), kvb.KvbRows: kvb.rows(-1, 1, 64, kvb.BF16), kvb.KvbList: kvb.KvbList(A, A, A, A, -1, 1)}
    args[0] = bad[type(args[0])]
    fn = getattr(kvb, name)
    assert fn(*args, stream=0, check=False) == kvb.EINVAL
    for i, a in enumerate(args):
        if a is A:
            with pytest.raises((TypeError, AttributeError)):
                fn(*args[:i], kvb.KvbShape(), *args[i + 1:], stream=0, check=False)
