"""kvb_scan against the fp64 recurrence: lengths around the chunks' edges, ragged batches, slots, strides, decays, refusals."""
import numpy as np
import pytest
import torch

from oracle import gdn as oracle
from paper_2605_19049_amd import kvb, synth
from harness import DT, TORCH_DT, UNIT, dev, host, rel_err

pytestmark = pytest.mark.gpu

# Largest error over the RMS.  Every factor of every product is held to 2^-24 and sums are fp32, as in the all-fp32 configuration
# of the other calls, whose bound this is: a few hundred roundings of 6e-8 that add up like a random walk.
TOL = 1e-5


class Seqs:
    """Ragged synthetic sequences in numpy (padded, as the oracle takes them) and packed on the GPU."""

    def __init__(self, lens, Hk, Hv, d, in_dtype, seed=0, g_lo=-0.5, gap=0, fused=False, spare=2):
        rng = np.random.default_rng(seed)
        self.lens, self.Hk, self.Hv, self.d, self.in_dtype = list(lens), Hk, Hv, d, in_dtype
        B, L = len(lens), max(1, max(lens))
        self.B, self.N = B, sum(lens) + gap
        x = synth.token_stream(rng, B, L, Hk, Hv, d, d, in_dtype)
        x["g"] = np.float32(rng.uniform(g_lo, 0.0, x["g"].shape) if g_lo else np.zeros(x["g"].shape))
        x["beta"] = np.float32(x["beta"])
        self.x = x
        self.starts = np.concatenate([[gap], gap + np.cumsum(lens)]).astype(np.int32)
        self.n_slots = B + spare
        self.slots = rng.permutation(self.n_slots)[:B].astype(np.int32)
        self.S = rng.standard_normal((self.n_slots, Hv, d, d)).astype(np.float32) * 0.5
        if fused:   # parts of the rows of one projection
            rows = torch.full((self.N, (2 * Hk + Hv) * d + 16), float("nan"), dtype=TORCH_DT[in_dtype], device="cuda")
            q, k, v = (p.view(self.N, -1, d) for p in rows[:, 8:-8].split([Hk * d, Hk * d, Hv * d], dim=1))
            q.copy_(self.pack(x["q"])), k.copy_(self.pack(x["k"])), v.copy_(self.pack(x["v"]))
            self.q, self.k, self.v = q, k, v
        else:
            self.q, self.k, self.v = (self.pack(x[n]) for n in "qkv")
        self.g, self.beta = self.pack(x["g"], False), self.pack(x["beta"], False)
        self.start, self.slot = dev(self.starts), dev(self.slots)
        self.state0 = dev(self.S)

    def pack(self, x, typed=True):
        y = np.full((self.N,) + x.shape[2:], np.nan, np.float32)
        for b, n in enumerate(self.lens):
            y[self.starts[b]:self.starts[b] + n] = x[b, :n]
        return dev(y, self.in_dtype if typed else None)

    def unpack(self, y, b):
        return y[self.starts[b]:self.starts[b] + self.lens[b]]

    def shape(self, out_dtype="f32", scale=0.125, B=None):
        return kvb.shape(self.B if B is None else B, self.Hk, self.Hv, self.d, self.d, 1, DT[self.in_dtype], scale=scale, out_dtype=DT[out_dtype])

    def seqs(self, slot=True):
        return kvb.seqs(self.start, self.N, self.n_slots, slot=self.slot if slot else None, q=self.q, k=self.k, v=self.v)

    def scan(self, out_dtype="f32", state0=True, state1=None, stream=None):
        sh, sq = self.shape(out_dtype), self.seqs()
        out = torch.full((self.N, self.Hv, self.d), 7.0, dtype=TORCH_DT[out_dtype], device="cuda")
        state1 = torch.full_like(self.state0, 7.0) if state1 is None else state1
        work = torch.full((kvb.scan_work(sh, sq) // 4,), float("nan"), device="cuda")
        kvb.kvb_scan(sh, sq, self.q, self.k, self.v, self.g, self.beta, self.state0 if state0 else None, state1, out, work, stream=stream)
        return out, state1

    def expected(self, state0=True, scale=0.125):
        S0 = self.S[self.slots] if state0 else np.zeros_like(self.S[self.slots])
        o, _, S, _ = oracle.gdn_sequence(S0, *(self.x[n] for n in ("q", "k", "v", "g", "beta")), scale, lens=self.lens)
        return o, S

    def check(self, out, state1, o, S, out_dtype="f32", tol=TOL):
        got, want = host(out), np.concatenate([o[b, :n] for b, n in enumerate(self.lens)])
        s1 = host(state1)
        if want.size:
            assert rel_err(got[self.starts[0]:], want, UNIT[out_dtype]) < tol
        assert rel_err(s1[self.slots], S) < tol
        assert (got[:self.starts[0]] == 7.0).all()
        spare = np.setdiff1d(np.arange(self.n_slots), self.slots)
        assert (s1[spare] == 7.0).all()


CASES = [
    # lengths, Hk, Hv, d, inputs, outputs
    ([1], 1, 1, 128, "bf16", "f32"), ([2, 1, 1, 3], 2, 4, 128, "bf16", "bf16"), ([63], 2, 2, 128, "bf16", "f32"),
    ([64], 2, 2, 128, "bf16", "f32"), ([65, 0, 17, 128], 2, 4, 128, "bf16", "f32"), ([0, 0, 5], 1, 3, 128, "bf16", "f32"),
    ([0], 1, 1, 128, "bf16", "f32"), ([1000], 1, 2, 128, "bf16", "bf16"), ([129, 300, 31, 16, 33, 48], 4, 8, 128, "bf16", "f32"),
    ([15, 100], 2, 4, 128, "f16", "f16"), ([200, 64], 1, 2, 128, "f16", "f32"), ([70, 130, 1], 1, 2, 128, "f32", "f32"),
    ([70, 130, 1], 3, 9, 64, "bf16", "bf16"), ([191], 2, 4, 64, "f16", "f32"), ([100, 257], 1, 2, 64, "f32", "f32"),
    ([70, 130, 1], 2, 4, 32, "bf16", "f32"), ([17, 99], 2, 2, 32, "f16", "f16"), ([100, 64, 63], 1, 2, 32, "f32", "f32"),
    ([3] * 70 + [130], 1, 1, 32, "bf16", "f32"),   # more sequences than lanes
]


@pytest.mark.parametrize("lens, Hk, Hv, d, in_dtype, out_dtype", CASES)
def test_against_the_recurrence(lens, Hk, Hv, d, in_dtype, out_dtype):
    t = Seqs(lens, Hk, Hv, d, in_dtype, seed=len(lens) + d)
    t.check(*t.scan(out_dtype), *t.expected(), out_dtype)


@pytest.mark.parametrize("in_dtype, d", [("bf16", 128), ("f16", 64), ("f32", 128)])
def test_rows_of_one_projection_and_a_gap_in_front(in_dtype, d):
    t = Seqs([90, 0, 64, 7], 2, 4, d, in_dtype, seed=3, gap=37, fused=True)
    t.check(*t.scan(), *t.expected())


@pytest.mark.parametrize("in_dtype", ["bf16", "f32"])
def test_no_first_state_and_in_place(in_dtype):
    t = Seqs([90, 0, 64, 7], 2, 4, 64, in_dtype, seed=4)
    t.check(*t.scan(state0=False), *t.expected(state0=False))
    o, S = t.expected()
    inplace = t.state0.clone()
    t.state0 = inplace
    out, s1 = t.scan(state1=inplace)
    assert rel_err(host(s1)[t.slots], S) < TOL
    assert rel_err(host(out), np.concatenate([o[b, :n] for b, n in enumerate(t.lens)])) < TOL


@pytest.mark.parametrize("g_lo", [0.0, -0.01, -30.0, -1000.0])
def test_decays_of_all_sizes(g_lo):
    """No decay at all, nearly none, and decays whose sums over a chunk are beyond what fp32 could take differences of."""
    t = Seqs([300, 64], 1, 2, 128, "bf16", seed=5, g_lo=g_lo)
    t.check(*t.scan(), *t.expected())


def test_minus_infinity_forgets_the_state():
    t = Seqs([100, 80], 1, 2, 64, "f32", seed=6)
    at = [(0, 0), (0, 64), (0, 77), (1, 30)]
    for b, i in at:
        t.x["g"][b, i] = -np.inf
    t.g = t.pack(t.x["g"], False)
    got = t.scan()
    for b, i in at:
        t.x["g"][b, i] = -1e4   # (exp is zero all the same; the oracle takes finite numbers)
    t.check(*got, *t.expected())


def test_pieces_of_a_sequence_give_the_whole():
    """A sequence in pieces of 1, 63, 64, 65 and 107 tokens, each from the state that the one before left."""
    t = Seqs([300], 2, 4, 128, "bf16", seed=7)
    o, S = t.expected()
    state, outs, at = t.state0.clone(), [], 0
    for n in (1, 63, 64, 65, 107):
        start = dev(np.array([at, at + n], np.int32))
        sh, sq = t.shape(), kvb.seqs(start, t.N, t.n_slots, slot=t.slot)
        out = torch.empty((t.N, t.Hv, t.d), device="cuda")
        work = torch.empty(kvb.scan_work(sh, sq), dtype=torch.uint8, device="cuda")
        kvb.kvb_scan(sh, sq, t.q, t.k, t.v, t.g, t.beta, state, state, out, work)
        outs.append(host(out)[at:at + n])
        at += n
    assert rel_err(np.concatenate(outs), o[0]) < TOL and rel_err(host(state)[t.slots], S) < TOL


def test_same_bits_every_time_and_on_another_stream():
    t = Seqs([90, 0, 640, 7], 2, 4, 128, "bf16", seed=8)
    out, s1 = t.scan("bf16")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out2, s2 = t.scan("bf16", stream=side)
    side.synchronize()
    assert torch.equal(out, out2) and torch.equal(s1, s2)


def test_a_bad_value_stays_in_its_sequence_and_behind_its_chunk():
    t = Seqs([200, 150], 1, 2, 64, "bf16", seed=9)
    clean, _ = t.scan()
    t.v[70, 0, 3] = float("inf")   # second chunk of the first sequence, head 0
    t.k[200 + 140, 0, 5] = float("nan")
    out, s1 = t.scan()
    o, c = host(out), host(clean)
    assert np.array_equal(o[:64], c[:64]) and np.array_equal(o[:200, 1], c[:200, 1]) and np.array_equal(o[200:328], c[200:328])
    assert not np.isfinite(o[70:200, 0, 3]).any() and np.isfinite(o[:200, 0, 40]).all()
    assert not np.isfinite(o[340:]).all()


def test_bounds_and_slots_that_make_no_sense_are_cut_off():
    t = Seqs([100, 80], 1, 2, 64, "bf16", seed=10)
    ref, _ = t.scan()
    t.start = dev(np.array([-50, 100, 10 ** 6], np.int32))
    out, s1 = t.scan()
    assert torch.equal(out, ref)
    t.start = dev(np.array([100, 40, 180], np.int32))   # descending: the first is empty
    out, s1 = t.scan()
    assert torch.equal(s1[t.slots[0]], t.state0[t.slots[0]])
    t.start, t.slot = dev(t.starts), dev(np.array([-1, t.n_slots], np.int32))
    out, s1 = t.scan()
    assert (host(out) == 7.0).all() and (host(s1) == 7.0).all()


def test_replayed_from_a_graph():
    t = Seqs([90, 0, 64, 7], 2, 4, 128, "bf16", seed=11)
    sh, sq = t.shape(), t.seqs()
    out, s1 = torch.zeros((t.N, t.Hv, t.d), device="cuda"), torch.zeros_like(t.state0)
    work = torch.empty(kvb.scan_work(sh, sq), dtype=torch.uint8, device="cuda")

    def call():
        kvb.kvb_scan(sh, sq, t.q, t.k, t.v, t.g, t.beta, t.state0, s1, out, work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(3):
        t.v.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want, ws = t.scan()
        assert torch.equal(out, want) and torch.equal(s1[t.slots], ws[t.slots])


def test_on_from_the_state_with_the_other_calls():
    """A prompt by kvb_scan, the next tokens by kvb_decode_flush."""
    t = Seqs([150, 90], 2, 4, 128, "bf16", seed=12, spare=1)
    n, B = 20, 2
    o, S = t.expected()
    ds = kvb.DeviceStore(t.n_slots, t.Hk, t.Hv, t.d, t.d, 8, kvb.BF16)
    out, _ = t.scan(state1=ds.state)
    more = synth.token_stream(np.random.default_rng(99), B, n, t.Hk, t.Hv, t.d, t.d, "bf16")
    want, _, S2, _ = oracle.gdn_sequence(S, *(more[x] for x in ("q", "k", "v", "g", "beta")), 0.125)
    sh = kvb.shape(B, t.Hk, t.Hv, t.d, t.d, 8, kvb.BF16, scale=0.125)
    got = torch.empty((n, B, t.Hv, t.d), device="cuda")
    for i in range(n):
        x = [dev(more[m][:, i], "bf16" if m in "qkv" else None) for m in ("q", "k", "v")] + \
            [dev(np.float32(more[m][:, i])) for m in ("g", "beta")]
        kvb.kvb_decode_flush(sh, ds.c(), t.slot, *x, got[i], 8)
    assert rel_err(host(got).transpose(1, 0, 2, 3), want) < 2e-4   # (the guard of the other calls)


def test_offsets_beyond_32_bits():
    """Rows of a projection so wide that the last tokens lie more than 2^32 bytes behind the first."""
    n, d, wide = 70, 32, 1 << 25   # elements from row to row: 64 MiB
    rows = torch.zeros((n * wide + 3 * d,), dtype=torch.bfloat16, device="cuda")
    t = Seqs([n], 1, 1, d, "bf16", seed=13, spare=0)
    views = [torch.as_strided(rows, (n, 1, d), (wide, d, 1), i * d) for i in range(3)]
    for to, x in zip(views, (t.q, t.k, t.v)):
        to.copy_(x)
    want = t.scan()
    t.q, t.k, t.v = views
    got = t.scan()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
