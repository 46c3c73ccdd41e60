"""What kvb_conv and its forms, kvb_norm, kvb_grad_norm and kvb_clip refuse before anything reaches the GPU, and how much workspace they ask for."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2605_19049_amd import kvb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x1000   # a fake, well-aligned address
GOOD = dict(B=2, Hk=2, Hv=4, dk=64, dv=64, cap=1, in_dtype=kvb.BF16)
C = 8 * 64


def shape(**kw):
    return kvb.shape(**{**GOOD, **kw})


def taps(**kw):
    t = kvb.taps(A, width=4, A_log=A, dt_bias=A)
    for n, v in kw.items():
        setattr(t, n, v)
    return t


def seqs(**kw):
    return kvb.seqs(**{**dict(start=A, n_tokens=10, n_slots=2), **kw})


CONV = dict(x=A, a=A, b=A, state0=A, state1=A, q=A, k=A, v=A, g=A, beta=A)
BACK = dict(x=A, a=A, b=A, state0=A, dq=A, dk=A, dv=A, dg=A, dbeta=A, dstate1=A, dx=A, da=A, db=A, dweight=A, dbias=None, dA_log=A, ddt_bias=A, dstate0=2 * A, work=A)


def conv(sh=None, ta=None, sq=None, **kw):
    return kvb.kvb_conv(sh or shape(), ta or taps(), sq or seqs(), *{**CONV, **kw}.values(), stream=0, check=False)


def decode(sh=None, ta=None, slot=A, n_slots=2, **kw):
    return kvb.kvb_conv_decode(sh or shape(), ta or taps(), slot, n_slots, *{**CONV, **kw}.values(), stream=0, check=False)


def verify(sh=None, ta=None, slot=A, n_slots=2, T=4, parent=A, **kw):
    d = {**CONV, **kw}
    d["state"] = d.pop("state0")
    return kvb.kvb_conv_verify(sh or shape(), ta or taps(), slot, n_slots, T, parent, d["x"], d["a"], d["b"], d["state"], d["q"], d["k"], d["v"], d["g"], d["beta"],
                               stream=0, check=False)


def commit(sh=None, ta=None, slot=A, n_slots=2, T=4, path=A, accepted=A, x=A, state0=A, state1=A):
    return kvb.kvb_conv_commit(sh or shape(), ta or taps(), slot, n_slots, T, path, accepted, x, state0, state1, stream=0, check=False)


def back(sh=None, ta=None, sq=None, **kw):
    return kvb.kvb_conv_backward(sh or shape(), ta or taps(), sq or seqs(), *{**BACK, **kw}.values(), stream=0, check=False)


FORMS = [conv, decode, verify, commit, back]


@pytest.mark.parametrize("bad, code", [
    (dict(B=-1), kvb.EINVAL), (dict(Hk=0), kvb.EINVAL), (dict(Hk=3), kvb.EINVAL), (dict(dk=0), kvb.EINVAL), (dict(dk=96, dv=96), kvb.EUNSUPPORTED),
    (dict(dk=64, dv=128), kvb.EUNSUPPORTED), (dict(in_dtype=3), kvb.EUNSUPPORTED), (dict(Hk=1 << 16, Hv=1 << 18), kvb.EINVAL)])
def test_shapes(bad, code):
    for f in FORMS:
        assert f(sh=shape(**bad)) == code, f


@pytest.mark.parametrize("bad, code", [
    (dict(weight=None), kvb.EINVAL), (dict(weight=A + 2), kvb.EINVAL), (dict(bias=A + 8), kvb.EINVAL), (dict(A_log=A + 2), kvb.EINVAL), (dict(dt_bias=A + 1), kvb.EINVAL),
    (dict(x_stride=C - 8), kvb.EINVAL), (dict(x_stride=C + 4), kvb.EINVAL), (dict(x_stride=1 << 26), kvb.EINVAL), (dict(a_stride=3), kvb.EINVAL),
    (dict(b_stride=(1 << 26) + 1), kvb.EINVAL), (dict(width=0), kvb.EINVAL), (dict(width=1), kvb.EUNSUPPORTED), (dict(width=5), kvb.EUNSUPPORTED),
    (dict(flags=2), kvb.EINVAL), (dict(eps=0.0), kvb.EINVAL), (dict(eps=1e-31), kvb.EINVAL), (dict(eps=-1.0), kvb.EINVAL), (dict(eps=float("nan")), kvb.EINVAL), (dict(eps=float("inf")), kvb.EINVAL)])
def test_taps(bad, code):
    for f in FORMS:
        # (a bias goes with its gradient)
        assert (f(ta=taps(**bad), dbias=A) if f is back and "bias" in bad else f(ta=taps(**bad))) == code, f


def test_inputs_and_results():
    for f in (conv, decode, verify):
        for bad in (dict(x=None), dict(x=A + 8), dict(a=None), dict(b=None), dict(a=A + 1), dict(state0=A + 8), dict(q=None), dict(k=None), dict(v=None), dict(v=A + 8),
                    dict(g=None), dict(beta=None), dict(g=A + 2), dict(a=None, b=None), dict(a=None, b=None, g=None)):
            assert f(**bad) == kvb.EINVAL, (f, bad)
        for bad in (dict(A_log=None), dict(dt_bias=None)):
            assert f(ta=taps(**bad)) == kvb.EINVAL
    assert conv(state1=A + 4) == kvb.EINVAL and decode(state1=A + 4) == kvb.EINVAL
    for f in (decode, verify, commit):
        assert f(slot=None) == kvb.EINVAL and f(slot=A + 2) == kvb.EINVAL and f(n_slots=-1) == kvb.EINVAL
    for f in (verify, commit):
        assert f(T=0) == kvb.EINVAL and f(T=9) == kvb.EINVAL
    assert verify(parent=A + 2) == kvb.EINVAL
    for bad in (dict(accepted=None), dict(accepted=A + 2), dict(path=A + 2), dict(x=None), dict(state1=None), dict(state1=A + 8), dict(state0=A + 8)):
        assert commit(**bad) == kvb.EINVAL, bad


def test_sequences():
    for f in (conv, back):
        for bad in (dict(start=None), dict(start=A + 2), dict(n_tokens=-1), dict(n_slots=-1), dict(slot=A + 2)):
            assert f(sq=seqs(**bad)) == kvb.EINVAL, (f, bad)
        for n in "qkv":
            sq = seqs()
            setattr(sq, n + "_stride", 64)
            assert f(sq=sq) == kvb.EINVAL
    assert conv(sh=shape(Hk=1024, Hv=1024), sq=seqs(n_tokens=2 ** 31 - 1)) == kvb.EINVAL   # more units than a launch has


def test_calls_that_a_launch_does_not_hold():
    """2^32 threads: 64 for each 512 channels of up to 64 tokens (a sequence is as much as 8 more), of a token or draft, and for its gates"""
    small = dict(Hk=1, Hv=1, dk=32, dv=32)
    assert conv(sh=shape(B=2 ** 30 - 1, **small), sq=seqs(n_tokens=0)) == kvb.EINVAL
    assert conv(sh=shape(B=2 ** 29, **small)) == kvb.EINVAL
    assert decode(sh=shape(B=2 ** 25, **small)) == kvb.EINVAL
    assert verify(sh=shape(B=2 ** 23, **small)) == kvb.EINVAL
    assert commit(sh=shape(B=2 ** 25, **small)) == kvb.EINVAL
    assert norm(ro=rows(n_tokens=2 ** 24, heads=1, width=2056)) == kvb.EINVAL
    assert norm(ro=rows(n_tokens=2 ** 23, heads=1, width=8200)) == kvb.EINVAL


def test_gradients():
    for bad in (dict(x=None), dict(dq=None), dict(dk=A + 8), dict(dv=None), dict(dg=None), dict(dbeta=A + 2), dict(dstate1=A + 8), dict(dx=None), dict(dx=A + 8), dict(da=None),
                dict(db=None), dict(db=A + 1), dict(dweight=None), dict(dweight=A + 2), dict(dbias=A), dict(dA_log=None), dict(ddt_bias=None), dict(dstate0=A),
                dict(dstate0=A + 8), dict(work=None), dict(work=A + 8), dict(a=None, b=None), dict(a=None, b=None, dg=None, dbeta=None, da=None, db=None)):
        assert back(**bad) == kvb.EINVAL, bad
    assert back(ta=taps(bias=A)) == kvb.EINVAL   # a bias without its gradient


def test_no_requests_is_nothing():
    none = shape(B=0)
    for f in (conv, decode, verify, commit):
        assert f(sh=none) == kvb.OK
    # (tensors of no elements have no address)
    assert decode(sh=none, slot=None, x=None, a=None, b=None, q=None, k=None, v=None, g=None, beta=None) == kvb.OK
    assert commit(sh=none, slot=None, path=None, accepted=None, x=None) == kvb.OK
    assert conv(sq=seqs(n_tokens=0), sh=none, x=None, a=None, b=None, q=None, k=None, v=None, g=None, beta=None) == kvb.OK


def test_workspace_grows():
    """That of the largest call serves smaller ones"""
    def work(n, B, **kw):
        return kvb.conv_backward_work(shape(B=B), taps(**kw), seqs(n_tokens=n))
    assert work(0, 0) > 0
    for B in (1, 3, 100):
        at = [work(n, B) for n in list(range(0, 3000, 7)) + [10 ** 5, 10 ** 6, 2 ** 28]]
        assert at == sorted(at)
    at = [work(1000, B) for B in range(0, 3000, 11)]
    assert at == sorted(at) and at[-1] < 1 << 26
    assert kvb.lib().kvb_conv_backward_work(ctypes.byref(shape()), ctypes.byref(taps(width=9)), ctypes.byref(seqs())) == kvb.EUNSUPPORTED
    for width in (8, 128, 520, 1000, 2048, 2056, 16384):
        at = [kvb.norm_backward_work(kvb.rows(n, 2, width, kvb.BF16)) for n in list(range(0, 3000, 7)) + [10 ** 5, 10 ** 6]]
        assert at == sorted(at) and at[-1] <= 1 << 26


NORM = dict(x=A, res=A, gate=A, weight=A, sum=A, out=A)
NORM_BACK = dict(x=A, gate=A, weight=A, dout=A, dsum=A, dx=A, dres=A, dgate=A, dweight=A, work=A)


def rows(**kw):
    r = kvb.rows(5, 2, 64, kvb.BF16)
    for n, v in kw.items():
        setattr(r, n, v)
    return r


def norm(ro=None, **kw):
    return kvb.kvb_norm(ro or rows(), *{**NORM, **kw}.values(), stream=0, check=False)


def norm_back(ro=None, **kw):
    return kvb.kvb_norm_backward(ro or rows(), *{**NORM_BACK, **kw}.values(), stream=0, check=False)


@pytest.mark.parametrize("bad, code", [
    (dict(n_tokens=-1), kvb.EINVAL), (dict(heads=0), kvb.EINVAL), (dict(width=0), kvb.EINVAL), (dict(width=12), kvb.EINVAL), (dict(width=16392), kvb.EINVAL),
    (dict(dtype=3), kvb.EUNSUPPORTED), (dict(x_dtype=7), kvb.EUNSUPPORTED), (dict(x_dtype=kvb.F16), kvb.EUNSUPPORTED), (dict(dtype=kvb.F32, x_dtype=kvb.BF16), kvb.EUNSUPPORTED),
    (dict(eps=0.0), kvb.EINVAL), (dict(eps=1e-31), kvb.EINVAL), (dict(eps=float("nan")), kvb.EINVAL), (dict(eps=float("inf")), kvb.EINVAL), (dict(scale=float("inf")), kvb.EINVAL),
    (dict(x_stride=64), kvb.EINVAL), (dict(x_stride=132), kvb.EINVAL), (dict(gate_stride=129), kvb.EINVAL), (dict(gate_stride=1 << 26), kvb.EINVAL),
    (dict(n_tokens=2 ** 31 - 1), kvb.EINVAL), (dict(heads=1 << 20), kvb.EINVAL)])
def test_rows(bad, code):
    assert norm(rows(**bad)) == code and norm_back(rows(**bad)) == code


def test_arrays_of_a_norm():
    for bad in (dict(x=None), dict(x=A + 8), dict(res=A + 8), dict(gate=A + 2), dict(weight=None), dict(weight=A + 8), dict(sum=A + 4), dict(out=None), dict(out=A + 8), dict(res=None)):
        assert norm(**bad) == kvb.EINVAL, bad
    assert norm(rows(scale=0.5), res=None, sum=None) == kvb.EINVAL   # a scale without a residual
    for bad in (dict(x=None), dict(x=A + 8), dict(gate=None), dict(dgate=None), dict(weight=None), dict(dout=None), dict(dsum=A + 8), dict(dx=None), dict(dres=A + 8),
                dict(dgate=A + 8), dict(dweight=None), dict(dweight=A + 2), dict(work=None), dict(work=A + 8)):
        assert norm_back(**bad) == kvb.EINVAL, bad
    assert norm(rows(n_tokens=0)) == kvb.OK and norm(rows(n_tokens=0), x=None, res=None, gate=None, sum=None, out=None) == kvb.OK


def some_list(**kw):
    li = kvb.KvbList(A, A, A, A, 2, 3)
    for n, v in kw.items():
        setattr(li, n, v)
    return li


def test_lists():
    def total(li, norm=A, work=A):
        return kvb.kvb_grad_norm(li, norm, work, stream=0, check=False)

    def clip(li, to=None, norm=A, largest=1.0):
        return kvb.kvb_clip(li, to, norm, largest, stream=0, check=False)

    for bad in (dict(n=-1), dict(blocks=-1), dict(n=0), dict(data=None), dict(size=None), dict(type=None), dict(first=None), dict(data=A + 4), dict(size=A + 4), dict(type=A + 2),
                dict(first=A + 2)):
        assert total(some_list(**bad)) == kvb.EINVAL and clip(some_list(**bad)) == kvb.EINVAL, bad
        assert clip(some_list(), some_list(**bad)) == kvb.EINVAL, bad
    assert total(some_list(), norm=None) == kvb.EINVAL and total(some_list(), norm=A + 2) == kvb.EINVAL and total(some_list(), work=None) == kvb.EINVAL
    assert total(some_list(), work=A + 4) == kvb.EINVAL
    assert clip(some_list(), norm=None) == kvb.EINVAL
    for largest in (-1.0, float("nan")):
        assert clip(some_list(), largest=largest) == kvb.EINVAL
    assert clip(some_list(), some_list(n=3)) == kvb.EINVAL and clip(some_list(), some_list(blocks=4)) == kvb.EINVAL
    assert clip(some_list(blocks=0)) == kvb.OK


def test_tensor_lists():
    li = kvb.TensorList([torch.zeros(5), torch.zeros(kvb.LIST_BLOCK + 1, dtype=torch.bfloat16), torch.zeros(0), torch.zeros(2, 3, dtype=torch.float16)])
    assert li.blocks == 4 and li._first.tolist() == [0, 1, 3, 3, 4] and li._type.tolist() == [kvb.F32, kvb.BF16, kvb.F32, kvb.F16]
    assert li._size.tolist() == [5, kvb.LIST_BLOCK + 1, 0, 6] and li._data.tolist() == [t.data_ptr() for t in li.tensors]
    other = [torch.ones_like(t) for t in li.tensors]
    empty = kvb.KvbList(None, None, None, None, 0, 0)
    for i, t in enumerate((torch.zeros(4), torch.zeros(kvb.LIST_BLOCK + 2, dtype=torch.bfloat16), torch.zeros(1), torch.zeros(6))):   # another size or type
        with pytest.raises(ValueError, match="sizes or types"):
            kvb.kvb_clip(li.c(), kvb.TensorList(other[:i] + [t] + other[i + 1:]).c(), A, 1.0, stream=0)
    with pytest.raises(ValueError, match="sizes or types"):
        kvb.bind("kvb_clip", li.c(), kvb.TensorList(other[:3]).c(), A, 1.0, 0)
    assert kvb.kvb_clip(kvb.TensorList([], device="cpu").c(), empty, A, 1.0, stream=0) == kvb.OK
    for bad in (torch.zeros(3, dtype=torch.float64), torch.zeros(3, dtype=torch.int32), torch.zeros(4, 6)[:, ::2], torch.zeros(4, 6).t()):
        with pytest.raises(ValueError):
            kvb.TensorList([torch.zeros(2), bad])


def test_tensors_that_share_memory():
    """The same tensor twice would count twice and be cut twice"""
    flat = torch.zeros(100)
    for bad in ([flat, flat], [flat[:50], flat[49:]], [flat, torch.zeros(3), flat[10:20]]):
        with pytest.raises(ValueError, match="share memory"):
            kvb.TensorList(bad)
    kvb.TensorList([flat[:50], flat[50:], flat[10:10], flat[20:20]])   # parts, and parts of nothing
    li = kvb.TensorList([flat[:50], flat[50:]])
    fine, moved, swapped = kvb.TensorList([flat[:50], torch.zeros(50)]), kvb.TensorList([torch.zeros(50), flat[10:60]]), kvb.TensorList([flat[50:], flat[:50]])
    kvb.bind("kvb_clip", li.c(), fine.c(), A, 1.0, 0)
    kvb.bind("kvb_clip", li.c(), li.c(), A, 1.0, 0)
    kvb.bind("kvb_clip", li.c(), kvb.TensorList([flat[:50], flat[50:]]).c(), A, 1.0, 0)
    for to in (moved, swapped):
        with pytest.raises(ValueError, match="shares memory"):
            kvb.bind("kvb_clip", li.c(), to.c(), A, 1.0, 0)


def test_layouts():
    """Tensors that do not lie as the structs say are refused by name; those that do go through to the library (which refuses B = -1)"""
    N, Hk, Hv, d = 6, 2, 4, 64
    row = torch.zeros(N, 700, dtype=torch.bfloat16)
    good = dict(x=torch.zeros(N, C, dtype=torch.bfloat16), a=torch.zeros(N, Hv), b=torch.zeros(N, Hv), state0=torch.zeros(2, 3, C), state1=torch.zeros(2, 3, C),
                q=torch.zeros(N, Hk, d), k=torch.zeros(N, Hk, d), v=torch.zeros(N, Hv, d), g=torch.zeros(N, Hv), beta=torch.zeros(N, Hv))

    def call(ta=None, **kw):
        g = {**good, **kw}
        ta = ta or kvb.taps(A, width=4, A_log=A, dt_bias=A, x=good["x"], a=good["a"], b=good["b"])
        return kvb.kvb_conv(shape(B=-1), ta, kvb.seqs(A, N, 2, q=good["q"], k=good["k"], v=good["v"]), *g.values(), stream=0, check=False)

    assert call() == kvb.EINVAL
    assert call(x=good["x"].view(2, 3, C)) == kvb.EINVAL and call(x=good["x"].view(N, 8, 64)) == kvb.EINVAL
    strided = kvb.taps(A, width=4, A_log=A, dt_bias=A, x=row[:, :C], a=row[:, C:C + Hv], b=row[:, C + Hv:C + 2 * Hv])
    assert (strided.x_stride, strided.a_stride, strided.b_stride) == (700, 700, 700)
    assert call(strided, x=row[:, :C], a=row[:, C:C + Hv], b=row[:, C + Hv:C + 2 * Hv]) == kvb.EINVAL
    for bad in (dict(x=row[:, :C]), dict(a=row[:, :Hv]), dict(state0=torch.zeros(2, C, 3).transpose(1, 2)), dict(q=torch.zeros(N, d, Hk).transpose(1, 2)),
                dict(v=torch.zeros(N, 2 * Hv, d)[:, :Hv]), dict(g=torch.zeros(Hv, N).t()), dict(beta=torch.zeros(N, 2 * Hv)[:, ::2])):
        with pytest.raises(ValueError, match=next(iter(bad))):
            call(**bad)
    with pytest.raises(ValueError):
        call(strided)   # packed tensors, strides of a projection
    for bad in (row.t()[:C].t()[:, ::2], torch.zeros(C, N).t()):
        with pytest.raises(ValueError):
            kvb.taps(A, x=bad)
    x, gate = torch.zeros(N, 3, 64), torch.zeros(N, 6, 64)[:, 3:]
    ro = kvb.rows(N, 3, 64, kvb.F32, x=x, gate=gate)
    assert ro.gate_stride == 6 * 64
    ro.n_tokens = -1
    w = torch.zeros(64)
    assert kvb.kvb_norm(ro, x, None, gate, w, None, torch.zeros(N, 3, 64), stream=0, check=False) == kvb.EINVAL
    for bad in ((gate, None, gate, w, None, x), (x, None, x, w, None, x), (x, gate, gate, w, None, x), (x, None, gate, w, gate, x), (x, None, gate, w, None, gate)):
        with pytest.raises(ValueError):
            kvb.kvb_norm(ro, *bad, stream=0, check=False)


PROBE = r"""
#include <stdio.h>
#include <stddef.h>
#include "kvb.h"
int main(void)
{
    printf("%zu %zu %zu %zu\n", sizeof(kvb_taps), offsetof(kvb_taps, x_stride), offsetof(kvb_taps, width), offsetof(kvb_taps, eps));
    printf("%zu %zu %zu %zu\n", sizeof(kvb_rows), offsetof(kvb_rows, n_tokens), offsetof(kvb_rows, x_dtype), offsetof(kvb_rows, scale));
    printf("%zu %zu %zu\n", sizeof(kvb_list), offsetof(kvb_list, first), offsetof(kvb_list, blocks));
    printf("%d %d %d\n", KVB_CONV_UNIT, KVB_MAX_WIDTH, KVB_LIST_BLOCK);
    return 0;
}
"""


def test_structs_as_a_c_caller_sees_them(tmp_path):
    src, exe = tmp_path / "probe.c", tmp_path / "probe"
    src.write_text(PROBE)
    subprocess.check_call(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    got = [[int(x) for x in line.split()] for line in subprocess.check_output([str(exe)], text=True).splitlines()]
    t, r, li = kvb.KvbTaps, kvb.KvbRows, kvb.KvbList
    assert got == [[ctypes.sizeof(t), t.x_stride.offset, t.width.offset, t.eps.offset], [ctypes.sizeof(r), r.n_tokens.offset, r.x_dtype.offset, r.scale.offset],
                   [ctypes.sizeof(li), li.first.offset, li.blocks.offset], [kvb.CONV_UNIT, kvb.MAX_WIDTH, kvb.LIST_BLOCK]]


def test_workspace_of_a_norm_grows_with_the_list():
    """That of the largest list serves shorter ones, which a call cuts up finer"""
    def work(blocks):
        return kvb.grad_norm_work(kvb.KvbList(A, A, A, A, 1, blocks) if blocks else kvb.KvbList(None, None, None, None, 0, 0))
    at = [work(blocks) for blocks in list(range(3001)) + [10 ** 5, 10 ** 6]]
    assert at == sorted(at) and at[0] == 0 and at[-1] <= 8 * 10 ** 6
    # (each workgroup leaves 8 bytes: four a block below 512 blocks, one from there on)
    assert all(w >= 8 * blocks * (4 if blocks < 512 else 1) for blocks, w in enumerate(at[:3001]))


def test_lists_that_a_launch_does_not_hold():
    """256 threads a block"""
    for blocks in (2 ** 24, 2 ** 31 - 1):
        li = some_list(blocks=blocks)
        assert kvb.lib().kvb_grad_norm_work(ctypes.byref(li)) == kvb.EINVAL
        assert kvb.kvb_grad_norm(li, A, A, stream=0, check=False) == kvb.EINVAL and kvb.kvb_clip(li, None, A, 1.0, stream=0, check=False) == kvb.EINVAL
    assert kvb.grad_norm_work(some_list(blocks=2 ** 24 - 2)) == 8 * (2 ** 24 - 2)
