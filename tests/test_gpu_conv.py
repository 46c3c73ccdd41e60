"""kvb_conv, kvb_conv_decode, kvb_conv_verify and kvb_conv_commit against the formulas in 64 bits, token by token."""
import pytest
import torch

from paper_2605_19049_amd import kvb
from layer_reference import Conv, V, cat, f64, gates, softplus, zeros
from running_error import check

pytestmark = pytest.mark.gpu
TYPES = {"f32": (kvb.F32, torch.float32), "bf16": (kvb.BF16, torch.bfloat16), "f16": (kvb.F16, torch.float16)}
EPS = 1e-6
FILL = -77.0


class Case:
    """Inputs of sequences (or of T drafts of each request) on the GPU"""

    def __init__(self, lens, Hk, Hv, d, W, dtype, seed=0, fused=False, bias=False, n_slots=None, lead=0, tail=0, scale=1.0):
        gen = torch.Generator().manual_seed(seed)
        self.lens, self.Hk, self.Hv, self.d, self.W, self.C = lens, Hk, Hv, d, W, (2 * Hk + Hv) * d
        self.code, self.dt = TYPES[dtype]
        B, C, self.N = len(lens), self.C, lead + sum(lens) + tail
        self.n_slots = n_slots or B

        def rand(*size):
            return torch.randn(*size, generator=gen)

        x, a, b = (scale * rand(self.N, n) for n in (C, Hv, Hv))
        if fused:
            row = torch.empty(self.N, -(-(C + 24 + 2 * Hv) // 8) * 8, dtype=self.dt, device="cuda")
            self.x, self.a, self.b = row[:, :C], row[:, C + 24:][:, :Hv], row[:, C + 24:][:, Hv:2 * Hv]
        else:
            self.x, self.a, self.b = (torch.empty(self.N, n, dtype=self.dt, device="cuda") for n in (C, Hv, Hv))
        for to, y in ((self.x, x), (self.a, a), (self.b, b)):
            to.copy_(y)
        self.weight = (W ** -0.5 * rand(C, W)).to(self.dt).cuda()
        self.bias = rand(C).to(self.dt).cuda() if bias else None
        self.A_log, self.dt_bias = rand(Hv).cuda(), rand(Hv).cuda()
        self.state0 = rand(self.n_slots, W - 1, C).to(self.dt).cuda()
        self.slot = torch.randperm(self.n_slots, generator=gen)[:B].to(torch.int32).cuda()
        ends = [lead]
        for n in lens:
            ends.append(ends[-1] + n)
        self.ends, self.start = ends, torch.tensor(ends, dtype=torch.int32, device="cuda")
        self.sh = kvb.shape(B, Hk, Hv, d, d, 1, self.code)
        self.ta = self.taps()
        self.sq = kvb.seqs(self.start, self.N, self.n_slots, slot=self.slot)

    def taps(self, unit=True):
        return kvb.taps(self.weight, width=self.W, bias=self.bias, A_log=self.A_log, dt_bias=self.dt_bias, x=self.x, a=self.a, b=self.b, unit=unit, eps=EPS)

    def outs(self, strided=False):
        if strided:
            row = torch.full((self.N, self.C + 16), FILL, dtype=self.dt, device="cuda")
            q, k, v = (y.unflatten(1, (-1, self.d)) for y in row[:, :self.C].split([self.Hk * self.d, self.Hk * self.d, self.Hv * self.d], 1))
        else:
            q, k, v = (torch.full((self.N, h, self.d), FILL, dtype=self.dt, device="cuda") for h in (self.Hk, self.Hk, self.Hv))
        return [q, k, v] + [torch.full((self.N, self.Hv), FILL, device="cuda") for _ in range(2)]

    def conv_of(self, state, rows, unit=True):
        """Conv over the state's rows [W - 1, C] (None: zero) and the token rows with these numbers"""
        E = zeros(self.W - 1, self.C) if state is None else f64(state)
        return Conv(cat([E, f64(self.x[rows])], 0), self.weight, self.bias, 2 * self.Hk + self.Hv, 2 * self.Hk, self.d, EPS, unit)

    def check_tokens(self, outs, at, conv, pick=slice(None)):
        n = conv.n_out[pick]
        for got, (lo, hi), what in zip(outs, ((0, self.Hk), (self.Hk, 2 * self.Hk), (2 * self.Hk, 2 * self.Hk + self.Hv)), "qkv"):
            check(got[at], n[:, lo:hi], what)

    def check_gates(self, outs, at):
        rate, y, beta = gates(self.a[at], self.b[at], self.A_log, self.dt_bias)
        check(outs[3][at], rate * softplus(y), "g")
        check(outs[4][at], beta, "beta")


def run(c, state0=True, state1=True, strided=False, unit=True, gated=True, stream=None):
    o = c.outs(strided)
    s1 = torch.full_like(c.state0, FILL) if state1 is True else state1
    sq = kvb.seqs(c.start, c.N, c.n_slots, slot=c.slot, q=o[0], k=o[1], v=o[2])
    ab, gb = ((c.a, c.b), o[3:]) if gated else ((None, None), (None, None))
    kvb.kvb_conv(c.sh, c.taps(unit), sq, c.x, *ab, c.state0 if state0 is True else state0, s1, *o[:3], *gb, stream=stream)
    torch.cuda.synchronize()
    return o, s1


def check_sequences(c, o, s1, state0, skipped=(), unit=True, gated=True):
    """Outputs and last states of every sequence, and what belongs to none as it was"""
    touched, slots = torch.zeros(c.N, dtype=torch.bool), set()
    for b, n in enumerate(c.lens):
        row = int(c.slot[b])
        if b in skipped:
            continue
        slots.add(row)
        at = slice(c.ends[b], c.ends[b + 1])
        touched[at] = True
        state = None if state0 is None else state0[row]
        conv = c.conv_of(state, at, unit)
        if n:
            c.check_tokens(o, at, conv)
            if gated:
                c.check_gates(o, at)
        if s1 is not None:
            assert torch.equal(s1[row].cpu().double(), conv.E.v[n:])
    for y in o[:5 if gated else 3]:
        assert (y[~touched] == FILL).all()
    if s1 is not None:
        for row in set(range(c.n_slots)) - slots:
            assert (s1[row] == FILL).all()


LENS = [[1], [5], [1, 2, 3, 4, 0, 7], [33, 0, 64, 65, 1, 32, 31], [300], [0, 0, 2]]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("W, heads, d", [(4, (2, 4), 128), (3, (3, 9), 64), (2, (1, 1), 32), (4, (5, 5), 32)])
def test_sequences(lens, W, heads, d, dtype):
    c = Case(lens, *heads, d, W, dtype, seed=len(lens), bias=W != 4)
    o, s1 = run(c)
    check_sequences(c, o, s1, c.state0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_one_projection_and_rows_of_no_sequence(dtype):
    """x, a and b inside wider rows, q, k and v too; tokens ahead of and behind the sequences, states of nobody, stay as they were"""
    c = Case([40, 3, 0, 17], 2, 4, 128, 4, dtype, fused=True, n_slots=9, lead=5, tail=11)
    o, s1 = run(c, strided=True)
    check_sequences(c, o, s1, c.state0)


def test_large_calls():
    """Longer pieces, and above 64 MiB x past the caches"""
    c = Case([4100, 1, 0, 2000, 31], 8, 16, 128, 4, "bf16", seed=3)
    big = Case([8000, 1, 0, 3000, 31], 8, 16, 128, 4, "bf16", seed=3)
    assert c.N * c.C * 2 <= 64 << 20 < big.N * big.C * 2
    for c in (c, big):
        o, s1 = run(c)
        # (the formulas for some stretches: whole sequences in 64 bits with bounds take long)
        for b, lo, hi in ((0, 0, 70), (0, c.lens[0] - 70, c.lens[0]), (1, 0, 1), (3, 0, 40), (3, c.lens[3] - 33, c.lens[3]), (4, 0, 31)):
            first, W = c.ends[b], c.W
            E = f64(c.state0[int(c.slot[b])]) if lo < W - 1 else V(torch.zeros(0, c.C, dtype=torch.float64))
            rows = cat([E, f64(c.x[first + max(0, lo - (W - 1)):first + hi])], 0)
            conv = Conv(rows, c.weight, c.bias, 2 * c.Hk + c.Hv, 2 * c.Hk, c.d, EPS)
            c.check_tokens(o, slice(first + lo, first + hi), conv)
            c.check_gates(o, slice(first + lo, first + hi))
        for b, n in enumerate(c.lens):
            want = torch.cat([c.state0[int(c.slot[b])], c.x[c.ends[b]:c.ends[b + 1]]])[-(c.W - 1):]
            assert torch.equal(s1[int(c.slot[b])], want)


@pytest.mark.parametrize("W, dtype", [(4, "bf16"), (3, "f16"), (2, "bf16"), (4, "f32")])
def test_the_same_bits_in_calls_of_any_size(W, dtype):
    """Above 100 MiB (in 16 bits) x is asked for in another way, and in each form a call is cut up as it fits"""
    c = Case([9000, 1, 0, 5000, 31], 8, 16, 128, W, dtype, seed=4, bias=W == 2)
    assert c.N * c.C * 2 > 100 << 20
    o, s1 = run(c)
    starts, slots = c.start, c.slot
    for b in range(5):
        c.start, c.slot = starts[b:b + 2].contiguous(), slots[b:b + 1].contiguous()
        c.sh, c.sq = kvb.shape(1, c.Hk, c.Hv, c.d, c.d, 1, c.code), kvb.seqs(c.start, c.N, c.n_slots, slot=c.slot)
        mine, state = run(c)
        at, row = slice(c.ends[b], c.ends[b + 1]), int(slots[b])
        assert all(torch.equal(x[at], y[at]) for x, y in zip(o, mine)) and torch.equal(s1[row], state[row])
    # a call of no more tokens than the sequence has
    c.x, c.a, c.b, c.N = (*(y[c.ends[3]:c.ends[4]] for y in (c.x, c.a, c.b)), 5000)
    c.start, c.slot = torch.tensor([0, 5000], dtype=torch.int32, device="cuda"), slots[3:4].contiguous()
    c.sq = kvb.seqs(c.start, c.N, c.n_slots, slot=c.slot)
    mine, state = run(c)
    at, row = slice(c.ends[3], c.ends[4]), int(slots[3])
    assert all(torch.equal(x[at], y) for x, y in zip(o, mine)) and torch.equal(s1[row], state[row])


def test_state_in_place_and_none():
    for lens in ([2], [1, 0, 3, 100]):
        c = Case(lens, 2, 2, 64, 4, "bf16", seed=7)
        before = c.state0.clone()
        o, s1 = run(c, state1=c.state0)
        check_sequences(c, o, s1, before)
        o, _ = run(c, state0=None, state1=None)
        check_sequences(c, o, None, None)
        o, s1 = run(c, state0=None)
        check_sequences(c, o, s1, None)


def test_pieces_of_a_sequence_one_after_the_other():
    """A prompt in three calls gives the bits that one call gives"""
    c = Case([101], 2, 4, 128, 4, "bf16", seed=9)
    whole, s_whole = run(c)
    o, state = c.outs(), c.state0.clone()
    for lo, hi in ((0, 2), (2, 50), (50, 101)):
        start = torch.tensor([lo, hi], dtype=torch.int32, device="cuda")
        kvb.kvb_conv(c.sh, c.ta, kvb.seqs(start, c.N, 1, slot=c.slot), c.x, c.a, c.b, state, state, *o)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(o, whole)) and torch.equal(state, s_whole)


def test_without_unit_and_without_gates():
    c = Case([9, 40], 2, 4, 64, 4, "f16", seed=4)
    o, s1 = run(c, unit=False, gated=False)
    check_sequences(c, o, s1, c.state0, unit=False, gated=False)
    assert all((y == FILL).all() for y in o[3:])


def test_slots_outside_and_bounds_that_do_not_ascend():
    c = Case([10, 20, 30], 1, 2, 128, 4, "bf16", n_slots=4)
    c.slot = torch.tensor([2, -1, 1], dtype=torch.int32, device="cuda")
    o, s1 = run(c)
    check_sequences(c, o, s1, c.state0, skipped=(1,))
    c.slot = torch.tensor([0, 4, 3], dtype=torch.int32, device="cuda")
    o, s1 = run(c)
    check_sequences(c, o, s1, c.state0, skipped=(1,))
    # cut off to 0 .. n_tokens and to lengths of zero: sequences 0 and 2 are as they say, 1 is empty
    c.slot = torch.tensor([0, 1, 3], dtype=torch.int32, device="cuda")
    c.lens, c.ends, c.start = [30, 0, 30], [0, 30, 30, 60], torch.tensor([-5, 30, 30, 1000], dtype=torch.int32, device="cuda")
    o, s1 = run(c)
    check_sequences(c, o, s1, c.state0)


def test_zero_rows_and_values_that_are_not_finite():
    """A row of zeros has queries of zero (eps); a value that is not finite reaches its head in its own and the next W - 1 tokens only"""
    c = Case([50], 2, 2, 64, 4, "bf16", seed=5)
    c.x[10:20] = 0
    c.x[30, 5] = float("inf")
    c.x[40, 2 * 2 * 64 + 7] = float("nan")   # a value's channel: no norm
    o, _ = run(c)
    assert (o[0][13:20] == 0).all() and (o[2][13:20] == 0).all()
    bad = [~torch.isfinite(y) for y in o]
    want = [torch.zeros_like(y) for y in bad]
    want[0][30:34, 0] = True
    want[2][40:44, 0, 7] = True
    assert torch.isfinite(o[3]).all()
    for y, w in zip(bad, want):
        assert not (y & ~w).any()
    assert bad[2][40:44, 0, 7].all() and bad[0][30].any()


@pytest.mark.parametrize("scale", [30.0, 1e-4])
def test_large_and_small_inputs(scale):
    c = Case([20, 5], 2, 4, 32, 4, "f32", seed=6, scale=scale)
    o, s1 = run(c)
    check_sequences(c, o, s1, c.state0)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("B, W, heads, d", [(1, 4, (16, 32), 128), (7, 3, (3, 9), 64), (70, 2, (1, 2), 32), (3, 4, (5, 5), 128)])
def test_single_tokens(B, W, heads, d, dtype):
    """kvb_conv_decode, and the same as sequences of one token; the state in place"""
    c = Case([1] * B, *heads, d, W, dtype, seed=B, fused=True, bias=W == 3, n_slots=B + 2)
    o, s1 = run(c)
    mine, state = c.outs(), c.state0.clone()
    kvb.kvb_conv_decode(c.sh, c.ta, c.slot, c.n_slots, c.x, c.a, c.b, state, state, *mine)
    torch.cuda.synchronize()
    check_sequences(c, mine, None, c.state0)
    assert all(torch.equal(x, y) for x, y in zip(mine, o))
    for row in range(c.n_slots):
        assert torch.equal(state[row], s1[row] if row in c.slot.tolist() else c.state0[row])
    # no state: zero, and none wanted
    kvb.kvb_conv_decode(c.sh, c.ta, c.slot, c.n_slots, c.x, c.a, c.b, None, None, *mine)
    torch.cuda.synchronize()
    check_sequences(c, mine, None, None)


@pytest.mark.parametrize("B", [64, 65, 200, 4096, 4097, 5000])
def test_many_sequences(B):
    """Sequences of one token or none, found among up to thousands: what kvb_conv_decode gives for those that have one"""
    lens = [0 if b % 7 == 3 else 1 for b in range(B)]
    c = Case(lens, 1, 2, 32, 4, "f32", seed=B, bias=True)
    o, s1 = run(c)
    some = torch.tensor([b for b in range(B) if lens[b]], device="cuda")
    mine, state = c.outs(), c.state0.clone()
    kvb.kvb_conv_decode(kvb.shape(len(some), 1, 2, 32, 32, 1, c.code), c.ta, c.slot[some].contiguous(), B, c.x, c.a, c.b, state, state, *mine)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(mine, o)) and torch.equal(s1, state)


def random_tree(T, gen):
    return [int(torch.randint(-1, i, (1,), generator=gen)) if i else -1 for i in range(T)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("T, W, heads, d", [(1, 4, (2, 4), 128), (2, 4, (2, 4), 64), (4, 3, (16, 32), 128), (8, 4, (3, 9), 32), (8, 2, (1, 2), 128)])
def test_drafts(T, W, heads, d, tree, dtype):
    """Outputs by root paths, the state as it was; then the commit of an accepted path, in place and apart"""
    B, gen = 6, torch.Generator().manual_seed(T)
    c = Case([T] * B, *heads, d, W, dtype, seed=T, fused=True, n_slots=B + 1)
    parent = [random_tree(T, gen) if tree else [i - 1 for i in range(T)] for _ in range(B)]
    pt = torch.tensor(parent, dtype=torch.int32, device="cuda")
    o, before = c.outs(), c.state0.clone()
    kvb.kvb_conv_verify(c.sh, c.ta, c.slot, c.n_slots, T, pt if tree else None, c.x, c.a, c.b, c.state0, *o)
    torch.cuda.synchronize()
    assert torch.equal(c.state0, before)
    c.check_gates(o, slice(0, c.N))
    paths, counts = torch.full((B, T), -1, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        for i in range(T):
            way, at = [], i
            while at >= 0:
                way, at = [b * T + at] + way, parent[b][at]
            c.check_tokens(o, slice(b * T + i, b * T + i + 1), c.conv_of(before[int(c.slot[b])], way), slice(len(way) - 1, len(way)))
            if i == (b + T) % (T + 1) - 1:   # none, the first, .. accepted
                counts[b] = len(way)
                paths[b, :len(way)] = torch.tensor(way) - b * T
    apart = torch.full_like(before, FILL)
    given = (c.slot, c.n_slots, T, paths.cuda() if tree else None, counts.cuda(), c.x)
    kvb.kvb_conv_commit(c.sh, c.ta, *given, before, apart)
    kvb.kvb_conv_commit(c.sh, c.ta, *given, c.state0, c.state0)
    torch.cuda.synchronize()
    for row in range(c.n_slots):
        b = c.slot.tolist().index(row) if row in c.slot.tolist() else None
        if b is None:
            assert (apart[row] == FILL).all() and torch.equal(c.state0[row], before[row])
            continue
        n = int(counts[b])
        drafts = [b * T + int(p) for p in paths[b, :n]] if tree else [b * T + i for i in range(n)]
        want = torch.cat([before[row], c.x[drafts]])[-(W - 1):]
        assert torch.equal(apart[row], want) and torch.equal(c.state0[row], want)


def test_bad_parents_paths_and_counts():
    """A parent outside -1 .. i-1 is the committed token; a path that does not ascend, or too long a one, commits nothing"""
    B, T, W = 6, 4, 4
    c = Case([T] * B, 2, 4, 64, W, "bf16", seed=8)
    odd = torch.tensor([[0, 1, 7, -3]] * B, dtype=torch.int32, device="cuda")
    flat = torch.tensor([[-1, -1, -1, -1]] * B, dtype=torch.int32, device="cuda")
    a, b = c.outs(), c.outs()
    for parent, o in ((odd, a), (flat, b)):
        kvb.kvb_conv_verify(c.sh, c.ta, c.slot, c.n_slots, T, parent, c.x, c.a, c.b, c.state0, *o)
    path = torch.tensor([[1, 0, -1, -1], [0, 0, -1, -1], [0, 4, -1, -1], [0, 1, 2, 3], [0, 1, 2, 3], [-1, 2, -1, -1]], dtype=torch.int32, device="cuda")
    count = torch.tensor([2, 2, 2, 5, -1, 2], dtype=torch.int32, device="cuda")
    s1 = torch.full_like(c.state0, FILL)
    kvb.kvb_conv_commit(c.sh, c.ta, c.slot, c.n_slots, T, path, count, c.x, c.state0, s1)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and torch.equal(s1, c.state0)
    # a slot outside is skipped
    c.slot[2] = 99
    o = c.outs()
    kvb.kvb_conv_verify(c.sh, c.ta, c.slot, c.n_slots, T, None, c.x, c.a, c.b, c.state0, *o)
    kvb.kvb_conv_commit(c.sh, c.ta, c.slot, c.n_slots, T, None, torch.full_like(count, 1), c.x, c.state0, c.state0)
    torch.cuda.synchronize()
    assert (o[0][2 * T:3 * T] == FILL).all() and not (o[0][3 * T:] == FILL).any()


def test_drafts_then_commit_are_single_tokens():
    """Three drafts of a chain, all accepted, leave what three calls for single tokens leave"""
    c = Case([3] * 5, 2, 4, 128, 4, "bf16", seed=11)
    o, state = c.outs(), c.state0.clone()
    kvb.kvb_conv_verify(c.sh, c.ta, c.slot, c.n_slots, 3, None, c.x, c.a, c.b, state, *o)
    kvb.kvb_conv_commit(c.sh, c.ta, c.slot, c.n_slots, 3, None, torch.full((5,), 3, dtype=torch.int32, device="cuda"), c.x, state, state)
    one = c.state0.clone()
    for t in range(3):
        rows = [y.view(5, 3, -1)[:, t].contiguous() for y in (c.x, c.a, c.b)]
        ta = kvb.taps(c.weight, width=4, A_log=c.A_log, dt_bias=c.dt_bias, eps=EPS)
        mine = [y.view((5, 3) + tuple(y.shape[1:]))[:, t].clone() for y in o]
        kvb.kvb_conv_decode(c.sh, ta, c.slot, c.n_slots, *rows, one, one, *mine)
        torch.cuda.synchronize()
        assert all(torch.equal(m, y.view((5, 3) + tuple(y.shape[1:]))[:, t]) for m, y in zip(mine, o))
    assert torch.equal(one, state)


def test_another_stream_and_a_replayed_graph():
    c = Case([70, 3], 2, 4, 128, 4, "bf16", seed=12)
    want, s_want = run(c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, s_got = run(c, stream=side)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(s_got, s_want)
    o, state = c.outs(), c.state0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvb.kvb_conv(c.sh, c.ta, c.sq, c.x, c.a, c.b, state, state, *o)
    for _ in range(3):
        before = state.clone()
        graph.replay()
        torch.cuda.synchronize()
        check_sequences(c, o, None, before)
        assert torch.equal(state[int(c.slot[0])], c.x[67:70])
        assert torch.equal(state[int(c.slot[1])], c.x[70:73])


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("T, W, heads, d", [(1, 4, (2, 4), 128), (2, 4, (2, 4), 64), (4, 3, (16, 32), 128), (8, 4, (3, 9), 32), (8, 2, (1, 2), 128)])
def test_drafts_in_fp16(T, W, heads, d, tree):
    test_drafts(T, W, heads, d, tree, "f16")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_drafts_are_written_as_single_tokens_are(dtype):
    """A chain of three, token by token into results that hold nothing yet: every element is written, with the bits of the drafts"""
    B, T = 5, 3
    c = Case([T] * B, 2, 4, 128, 4, dtype, seed=13, bias=True)
    o, state = c.outs(), c.state0.clone()
    kvb.kvb_conv_verify(c.sh, c.ta, c.slot, c.n_slots, T, None, c.x, c.a, c.b, state, *o)
    kvb.kvb_conv_commit(c.sh, c.ta, c.slot, c.n_slots, T, None, torch.full((B,), T, dtype=torch.int32, device="cuda"), c.x, state, state)
    one = c.state0.clone()
    ta = kvb.taps(c.weight, width=4, bias=c.bias, A_log=c.A_log, dt_bias=c.dt_bias, eps=EPS)
    for t in range(T):
        rows = [y.view(B, T, -1)[:, t].contiguous() for y in (c.x, c.a, c.b)]
        mine = [torch.full((B,) + tuple(y.shape[1:]), FILL, dtype=y.dtype, device="cuda") for y in o]
        kvb.kvb_conv_decode(c.sh, ta, c.slot, c.n_slots, *rows, one, one, *mine)
        torch.cuda.synchronize()
        for m, y in zip(mine, o):
            assert not (m == FILL).any() and torch.equal(m, y.view((B, T) + tuple(y.shape[1:]))[:, t])
    assert torch.equal(one, state)
