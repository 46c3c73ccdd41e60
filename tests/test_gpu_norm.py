"""kvb_norm and kvb_norm_backward against the formulas in 64 bits."""
import pytest
import torch

from paper_2605_19049_amd import kvb
from layer_reference import V, f64, norm, norm_backward
from running_error import check
from test_gpu_conv import FILL, TYPES

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Rows:
    def __init__(self, n, heads, width, dtype, x_dtype=None, gate=False, res=False, seed=0, strided=False, scale=None):
        gen = torch.Generator().manual_seed(seed)
        self.n, self.heads, self.width = n, heads, width
        (self.code, self.dt), (self.x_code, self.xt) = TYPES[dtype], TYPES[x_dtype or dtype]

        def rand(dt, wide=False):
            y = torch.randn(n, heads, width, generator=gen).to(dt)
            if not wide:
                return y.cuda()
            row = torch.full((n, heads * width + 24), FILL, dtype=dt, device="cuda")
            row[:, 8:8 + heads * width] = y.flatten(1).cuda()
            return row[:, 8:8 + heads * width].unflatten(1, (heads, width))

        self.x = rand(self.xt, strided)
        self.x.mul_(torch.randn(n, heads, 1, generator=gen).exp().to(self.xt).cuda())
        self.res = rand(self.xt) if res else None
        self.gate = rand(self.dt, strided) if gate else None
        self.weight = (1.0 + 0.3 * torch.randn(width, generator=gen)).to(self.dt).cuda()
        self.dout, self.dsum = rand(self.dt), rand(self.xt)
        self.scale = (0.75 if res else 1.0) if scale is None else scale
        self.ro = kvb.rows(n, heads, width, self.code, x_dtype=self.x_code, x=self.x, gate=self.gate, eps=EPS, scale=self.scale)

    def sum(self):
        """s and its bound; what is stored is s rounded"""
        if self.res is None:
            return f64(self.x)
        s = f64(self.res).v + self.scale * f64(self.x).v
        return V(s, s.abs() + (self.scale * f64(self.x).v).abs())


def forward(c, sum=True, stream=None):
    out = torch.full((c.n, c.heads, c.width), FILL, dtype=c.dt, device="cuda")
    s = torch.full((c.n, c.heads, c.width), FILL, dtype=c.xt, device="cuda") if c.res is not None and sum else None
    kvb.kvb_norm(c.ro, c.x, c.res, c.gate, c.weight, s, out, stream=stream)
    torch.cuda.synchronize()
    return s, out


def check_forward(c, s, out):
    if s is not None:
        check(s, c.sum(), "sum")
    # the norm is of the sum as its type holds it
    want, *_ = norm(f64(s) if s is not None else c.sum(), c.weight, c.gate, EPS)
    check(out, want, "out")


PAIRS = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]
KINDS = [(False, False), (True, False), (False, True), (True, True)]
SMALL = [(1, 1, 8), (1, 1, 2048), (3, 1, 40), (5, 4, 32), (70, 3, 64), (9, 2, 136), (4, 1, 520), (2, 1, 1000), (3, 1, 2056), (2, 1, 8192), (1, 1, 16384)]
LARGE = [(33, 32, 128), (1100, 1, 520), (1100, 1, 1032), (1030, 1, 2048), (2, 1, 4096), (2, 1, 8200)]
CASES = [s + k + p for s in SMALL for k in KINDS for p in PAIRS] + [s + KINDS[(i + j) % 4] + PAIRS[(2 * i + j) % 5] for i, s in enumerate(LARGE) for j in range(5)]


@pytest.mark.parametrize("n, heads, width, gate, res, dtype, x_dtype", CASES)
def test_forward(n, heads, width, gate, res, dtype, x_dtype):
    c = Rows(n, heads, width, dtype, x_dtype, gate, res, seed=n + width)
    check_forward(c, *forward(c))


def lies_as(y):
    """A tensor of FILL that lies as y does, inside rows of FILL"""
    if y.is_contiguous():
        return torch.full_like(y, FILL)
    row = torch.full((y.shape[0], y.stride(0)), FILL, dtype=y.dtype, device="cuda")
    return row[:, 8:8 + y.shape[1] * y.shape[2]].unflatten(1, tuple(y.shape[1:]))


def backward(c, dsum=True, dres=True, stream=None):
    r = {"dx": lies_as(c.x), "dres": torch.full((c.n, c.heads, c.width), FILL, dtype=c.xt, device="cuda") if dres else None,
         "dgate": lies_as(c.gate) if c.gate is not None else None,
         "dweight": torch.empty(c.width, device="cuda")}
    work = torch.empty(kvb.norm_backward_work(c.ro), dtype=torch.uint8, device="cuda")
    kvb.kvb_norm_backward(c.ro, c.x, c.gate, c.weight, c.dout, c.dsum if dsum else None, *r.values(), work, stream=stream)
    torch.cuda.synchronize()
    return r


def check_backward(c, r, dsum=True):
    # (a lane adds the rows of its turns, then lanes, waves and parts: at most that many rows' roundings and 100 more)
    rows = c.n * c.heads
    want = norm_backward(f64(c.x), c.weight, c.gate, EPS, c.dout, c.dsum if dsum else None, c.scale, 100 + rows // 1024)
    for n, y in r.items():
        if y is not None:
            check(y, want[n], n)


@pytest.mark.parametrize("n, heads, width, gate, res, dtype, x_dtype", CASES)
def test_backward(n, heads, width, gate, res, dtype, x_dtype):
    c = Rows(n, heads, width, dtype, x_dtype, gate, scale=0.75 if res else 1.0, seed=n + width)
    check_backward(c, backward(c, dsum=res, dres=res), dsum=res)


@pytest.mark.parametrize("n, heads, width", [(70, 4, 128), (1030, 1, 1000), (3, 2, 2056)])
def test_rows_that_lie_apart(n, heads, width):
    """x and gate inside wider rows; what lies between the rows stays"""
    c = Rows(n, heads, width, "bf16", gate=True, strided=True)
    check_forward(c, *forward(c))
    r = backward(c)
    check_backward(c, r)
    for y in (r["dx"], r["dgate"]):
        row = y._base
        assert (row[:, :8] == FILL).all() and (row[:, 8 + heads * width:] == FILL).all() and not (y == FILL).any()


@pytest.mark.parametrize("n, heads, width, gate, res", [(13000, 32, 64, True, False), (26000, 1, 1000, False, True), (7000, 1, 4096, False, True)])
def test_large_calls(n, heads, width, gate, res):
    """Above 96 MiB of x, residual and gate these pass the caches: the same bits as smaller calls give"""
    c = Rows(n, heads, width, "bf16", gate=gate, res=res)
    assert n * heads * width * 4 > 96 << 20
    s, out = forward(c)
    for lo in range(0, n, n // 3):
        hi, part = min(n, lo + n // 3), torch.empty_like(out[lo:lo + n // 3])
        sums = torch.empty_like(part) if res else None
        kvb.kvb_norm(kvb.rows(hi - lo, heads, width, c.code, eps=EPS, scale=c.scale), c.x[lo:hi], c.res[lo:hi] if res else None, c.gate[lo:hi] if gate else None, c.weight, sums, part)
        torch.cuda.synchronize()
        assert torch.equal(part, out[lo:hi]) and (not res or torch.equal(sums, s[lo:hi]))


@pytest.mark.parametrize("width", [64, 128, 1000, 2056])
def test_few_rows(width):
    """Up to four turns of a workgroup need no parts; a gradient that is not aligned to 16 bytes is summed from one all the same"""
    at_once = 256 // (width // 8) if width <= 128 else 512 // (-(-width // 512) * 64)
    for n in (1, at_once, at_once + 1, 4 * at_once - 1, 4 * at_once, 4 * at_once + 1):
        c = Rows(n, 1, width, "bf16", gate=True, seed=n)
        r = backward(c)
        check_backward(c, r)
        flat = torch.full((width + 8,), FILL, device="cuda")
        dx, dres, dgate = (torch.empty_like(c.x) for _ in range(3))
        kvb.kvb_norm_backward(c.ro, c.x, c.gate, c.weight, c.dout, c.dsum, dx, dres, dgate, flat[1:width + 1], torch.empty(kvb.norm_backward_work(c.ro), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(flat[1:width + 1], r["dweight"]) and flat[0] == FILL and (flat[width + 1:] == FILL).all() and torch.equal(dx, r["dx"])


def test_in_place():
    """The residual's stream in place; out over x and over the gate"""
    c = Rows(100, 1, 1024, "bf16", res=True)
    s, out = forward(c)
    stream, other = c.res.clone(), torch.empty_like(out)
    kvb.kvb_norm(c.ro, c.x, stream, None, c.weight, stream, other)
    assert torch.equal(stream, s) and torch.equal(other, out)
    x = c.x.clone()
    kvb.kvb_norm(c.ro, x, c.res, None, c.weight, x, other)
    assert torch.equal(x, s) and torch.equal(other, out)
    x = c.x.clone()
    kvb.kvb_norm(c.ro, x, c.res, None, c.weight, None, x)
    assert torch.equal(x, out)
    c = Rows(50, 8, 128, "f16", gate=True)
    _, out = forward(c)
    gate = c.gate.clone()
    kvb.kvb_norm(c.ro, c.x, None, gate, c.weight, None, gate)
    assert torch.equal(gate, out)
    c = Rows(64, 1, 256, "f32", scale=0.5)
    want = backward(c)
    dsum, dx, dweight = c.dsum.clone(), torch.empty_like(c.x), torch.empty(256, device="cuda")
    kvb.kvb_norm_backward(c.ro, c.x, None, c.weight, c.dout, dsum, dx, dsum, None, dweight,
                          torch.empty(kvb.norm_backward_work(c.ro), dtype=torch.uint8, device="cuda"))
    assert torch.equal(dsum, want["dres"]) and torch.equal(dx, want["dx"]) and torch.equal(dweight, want["dweight"])


def test_zero_rows_and_values_that_are_not_finite():
    for width in (128, 1000, 4096):
        c = Rows(6, 1, width, "bf16", gate=True)
        c.x[1] = 0
        c.x[2, 0, 5] = float("nan")
        c.x[3, 0, 6] = float("inf")
        c.gate[4, 0, 7] = float("nan")
        _, out = forward(c)
        assert (out[1] == 0).all() and torch.isnan(out[2]).all()
        assert torch.isnan(out[3, 0, 6]) and (out[3, 0, :6] == 0).all()   # infinity / infinity, and what it leaves of the others
        assert torch.isnan(out[4]).sum() == 1 and torch.isfinite(out[0]).all() and torch.isfinite(out[5]).all()


def test_gates_far_from_zero():
    """exp overflows and underflows: silu is z or 0, its slope 1 or 0"""
    c = Rows(8, 2, 64, "f32", gate=True)
    c.gate[0] = 300.0
    c.gate[1] = -300.0
    check_forward(c, *forward(c))
    check_backward(c, backward(c))


def test_no_rows():
    c = Rows(0, 4, 64, "bf16", gate=True)
    forward(c)
    assert (backward(c)["dweight"] == 0).all()


def test_the_same_bits_another_stream_and_a_replayed_graph():
    c = Rows(5000, 2, 128, "bf16", gate=True)
    want, (_, out) = backward(c), forward(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again, (_, other) = backward(c, stream=side), forward(c, stream=side)
    assert torch.equal(out, other) and all(torch.equal(want[n], again[n]) for n in want)
    r, o = {n: torch.empty_like(y) for n, y in want.items()}, torch.empty_like(out)
    work = torch.empty(kvb.norm_backward_work(c.ro), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvb.kvb_norm(c.ro, c.x, None, c.gate, c.weight, None, o)
        kvb.kvb_norm_backward(c.ro, c.x, c.gate, c.weight, c.dout, c.dsum, r["dx"], r["dres"], r["dgate"], r["dweight"], work)
    for _ in range(3):
        for y in list(r.values()) + [o, work]:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and all(torch.equal(want[n], r[n]) for n in want)


def turns(rows, width):
    """Turns that the rows take if each is a workgroup's, and rows of a turn"""
    if width <= 512:
        lanes = 4
        while lanes < 64 and 8 * lanes < width:
            lanes *= 2
        at_once = 256 // lanes
    else:
        vectors = 1 if width <= 4096 else 2 if width <= 8192 else 4
        at_once = 512 // (-(-(-(-width // 8 // vectors)) // 64) * 64)
    return -(-rows // at_once), at_once


MANY = [(8, 300), (32, 1100), (8, 12300), (128, 300), (120, 1100), (64, 2500), (512, 600), (520, 521), (2056, 530), (4096, 700)]


@pytest.mark.parametrize("dtype, x_dtype, gate", [("bf16", "f32", True), ("f16", "f16", False), ("f32", "f32", True)])
@pytest.mark.parametrize("width, want", MANY)
def test_gradients_of_many_turns(width, want, dtype, x_dtype, gate):
    """More turns than workgroups, the last one not full"""
    n = want * turns(1, width)[1] - (turns(1, width)[1] > 1)
    assert turns(n, width)[0] == want
    check_many(Rows(n, 1, width, dtype, x_dtype, gate=gate, seed=want))


@pytest.mark.parametrize("dtype, x_dtype, gate", [("bf16", "bf16", True), ("f16", "f32", False), ("f32", "f32", True)])
@pytest.mark.parametrize("n", [3, 5, 521])
@pytest.mark.parametrize("width", [4104, 8192, 8200, 16384])
def test_gradients_of_wide_rows(width, n, dtype, x_dtype, gate):
    """A workgroup a row, each with a part of the sums; the last of them with two rows"""
    assert turns(n, width) == (n, 1)
    check_many(Rows(n, 1, width, dtype, x_dtype, gate=gate, seed=n))


def check_many(c):
    """Additions on the way of a term of dweight: a lane's rows (turns / parts, at most 25 + rows / 1024), 4 waves of up to 16 rows, parts by 64 and then 64"""
    r = backward(c)
    want = norm_backward(f64(c.x), c.weight, c.gate, EPS, c.dout, c.dsum, c.scale, 25 + c.n * c.heads // 1024 + 64 + 16 + 64)
    for n, y in r.items():
        if y is not None:
            check(y, want[n], n)
