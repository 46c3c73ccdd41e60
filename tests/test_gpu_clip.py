"""kvb_grad_norm and kvb_clip against sums in 64 bits."""
import math

import pytest
import torch

from paper_2605_19049_amd import kvb

pytestmark = pytest.mark.gpu
B = kvb.LIST_BLOCK
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def some(sizes, types, seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=gen)).to(t).cuda() for n, t in zip(sizes, types)]


def norm_of(tensors):
    li = kvb.TensorList(tensors)
    norm = torch.full((1,), -1.0, device="cuda")
    kvb.kvb_grad_norm(li.c(), norm, torch.empty(kvb.grad_norm_work(li.c()), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    return li, norm


def want_norm(tensors):
    return math.sqrt(math.fsum(float(x.double().square().sum()) for x in tensors))


def check(tensors, largest):
    li, norm = norm_of(tensors)
    want = want_norm(tensors)
    assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.01   # one rounding, of a sum in 64 bits
    to = [torch.full_like(x, -77.0) for x in tensors]
    kvb.kvb_clip(li.c(), kvb.TensorList(to).c(), norm, largest)
    cut = min(1.0, largest / (want + 1e-6))
    before = [x.clone() for x in tensors]
    kvb.kvb_clip(li.c(), None, norm, largest)
    torch.cuda.synchronize()
    for x, y, z in zip(before, to, tensors):
        # norm, the sum with 1e-6, the quotient (2.5 units in the last place at most), the product; the last rounding
        f = torch.finfo(x.dtype)
        off, size = (y.double() - cut * x.double()).abs(), cut * x.double().abs()
        allowed = 8 * 2.0 ** -24 * size + (0 if x.dtype == torch.float32 else f.eps / 2) * size + f.smallest_normal * f.eps
        assert (off <= allowed).all()
        assert torch.equal(y, z)
        if cut == 1.0:
            assert torch.equal(x, y)


@pytest.mark.parametrize("largest", [1.0, 1e9])
@pytest.mark.parametrize("sizes", [[1], [7, 8, 9], [0, 5, 0, 0, 3, 0], [B], [B - 1, B + 1, 3 * B + 5, 1], [100003]], ids=str)
@pytest.mark.parametrize("shift", [0, 1, 2])
def test_sizes_and_types(sizes, shift, largest):
    check(some(sizes, [TYPES[(i + shift) % 3] for i in range(len(sizes))]), largest)


def test_many_tensors():
    sizes = [(i * 37) % 200 for i in range(1000)]
    check(some(sizes, [TYPES[i % 3] for i in range(1000)]), 2.0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("at, other", [(0, 0), (1, 1), (3, 3), (1, 2), (0, 5), (7, 0)])
def test_addresses_aligned_to_an_element_only(dtype, at, other):
    """Parts of a flat buffer, alike in their place among 16 bytes or not; what lies around them stays"""
    n = 2 * B + 77
    flat, flat_to = some([n + 20, n + 20], [dtype] * 2)
    x, to = flat[at:at + n], flat_to[other:other + n]
    kept = flat_to.clone()
    li, norm = norm_of([x])
    want = want_norm([x])
    assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.01
    kvb.kvb_clip(li.c(), kvb.TensorList([to]).c(), norm, 1.0)
    torch.cuda.synchronize()
    cut = torch.tensor(1.0, device="cuda") / (norm + 1e-6)
    # (a quotient that is rounded otherwise is off by 2.5 units at most)
    off = (to.double() - (x.float() * cut).double()).abs()
    assert (off <= (torch.finfo(dtype).eps + 3 * 2.0 ** -23) * x.double().abs() * float(cut) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps).all()
    assert torch.equal(flat_to[:other], kept[:other]) and torch.equal(flat_to[other + n:], kept[other + n:])


def test_large_values_and_small_ones():
    """Squares that fp32 does not hold"""
    big = [torch.tensor([3e30, 4e30], device="cuda"), torch.tensor([1e-30], device="cuda")]
    _, norm = norm_of(big)
    assert abs(float(norm) - 5e30) < 1e24
    small = [torch.tensor([3e-30, 4e-30], device="cuda")]
    _, norm = norm_of(small)
    assert abs(float(norm) - 5e-30) < 1e-36


def test_norms_that_are_not_finite():
    x = some([100], [torch.float32])[0]
    for value, finite in ((float("inf"), True), (float("nan"), False)):
        y = x.clone()
        y[3] = value
        li, norm = norm_of([y])
        assert not torch.isfinite(norm).any()
        kvb.kvb_clip(li.c(), None, norm, 1.0)
        torch.cuda.synchronize()
        assert torch.isnan(y[3])
        rest = torch.cat([y[:3], y[4:]])
        assert (rest == 0).all() if finite else torch.isnan(rest).all()


def test_nothing():
    for tensors in ([], some([0, 0], [torch.float32] * 2)):
        li, norm = norm_of(tensors)
        assert float(norm) == 0.0
        kvb.kvb_clip(li.c(), None, norm, 1.0)
    x = some([100], [torch.bfloat16])
    li, norm = norm_of(x)
    kvb.kvb_clip(li.c(), None, norm, 0.0)
    torch.cuda.synchronize()
    assert (x[0] == 0).all()


def test_another_stream_and_a_replayed_graph():
    tensors = some([50000, 3, 70001], TYPES)
    to = [torch.empty_like(x) for x in tensors]
    li, lt, norm = kvb.TensorList(tensors), kvb.TensorList(to), torch.empty(1, device="cuda")
    work = torch.empty(kvb.grad_norm_work(li.c()), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    kvb.kvb_grad_norm(li.c(), norm, work, stream=side)
    kvb.kvb_clip(li.c(), lt.c(), norm, 1.0, stream=side)
    side.synchronize()
    first = float(norm)
    assert abs(first - want_norm(tensors)) <= 2.0 ** -24 * first * 1.01
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvb.kvb_grad_norm(li.c(), norm, work)
        kvb.kvb_clip(li.c(), lt.c(), norm, 1.0)
    for i in range(3):
        for x in tensors:
            x.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = want_norm(tensors)
        assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.01
        assert abs(want_norm(to) - 1.0) < 0.004   # (bf16: each element is off by half a step of 2^-8 at most)


def test_one_workspace_for_lists_of_any_length():
    """The longest list's: one of 511 blocks, each of which leaves four sums, takes more of it than one of 600.  What lies behind stays"""
    tensors = some([i * 5 % 90 + 1 for i in range(600)], [TYPES[i % 3] for i in range(600)])
    room = kvb.grad_norm_work(kvb.TensorList(tensors).c())
    buffer = torch.full((room + 65536,), 119, dtype=torch.uint8, device="cuda")
    for n in (1, 127, 128, 511, 512, 600):
        li, norm = kvb.TensorList(tensors[:n]), torch.full((1,), -1.0, device="cuda")
        assert li.blocks == n
        kvb.kvb_grad_norm(li.c(), norm, buffer)
        torch.cuda.synchronize()
        want = want_norm(tensors[:n])
        assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.01
        assert (buffer[room:] == 119).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("at, other", [(0, 0), (1, 1), (5, 5), (1, 2), (0, 7)])
def test_whole_blocks(dtype, at, other):
    """Lists of 512 blocks and more have a workgroup for 16384 elements: parts of a flat buffer, at any element of it, with something between them that stays"""
    sizes = [5_000_077, 3 * B, 3_400_001, B - 1, B, B + 1, 9, 14336, 14337 + 7 * B]
    flat, flat_to = some([sum(sizes) + 16 * len(sizes) + 16] * 2, [dtype] * 2)
    kept, kept_to = flat.clone(), flat_to.clone()

    def parts(buffer, first):
        out, p = [], first
        for n in sizes:
            out.append(buffer[p:p + n])
            p += n + 16   # (source and result of each lie alike among 16 bytes if those of the first do)
        return out
    tensors, to = parts(flat, at), parts(flat_to, other)
    li, norm = norm_of(tensors)
    assert li.blocks >= 512
    want = want_norm(tensors)
    assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.01
    kvb.kvb_clip(li.c(), kvb.TensorList(to).c(), norm, 1000.0)
    torch.cuda.synchronize()
    assert torch.equal(flat, kept)
    cut, f = 1000.0 / (want + 1e-6), torch.finfo(dtype)
    assert cut < 0.5
    for x, y in zip(tensors, to):
        # (as in check: norm, the sum with 1e-6, the quotient, the product; the last rounding)
        off, size = (y.double() - cut * x.double()).abs(), cut * x.double().abs()
        assert (off <= 8 * 2.0 ** -24 * size + (0 if dtype == torch.float32 else f.eps / 2) * size + f.smallest_normal * f.eps).all()
    between = torch.ones(len(flat), dtype=torch.bool, device="cuda")
    for x in parts(between, other):
        x.zero_()
    assert torch.equal(flat_to[between], kept_to[between])
    kvb.kvb_clip(li.c(), None, norm, 1000.0)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(tensors, to))
    between.fill_(True)
    for x in parts(between, at):
        x.zero_()
    assert torch.equal(flat[between], kept[between])
    # nothing to cut: in place as it is, elsewhere a copy
    kvb.kvb_clip(li.c(), None, norm, 1e9)
    kvb.kvb_clip(li.c(), kvb.TensorList(to).c(), norm, 1e9)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(tensors, to)) and torch.equal(flat[between], kept[between])
