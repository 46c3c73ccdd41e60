"""kvb_scan_backward against the fp64 gradients of the recurrence, and against differences of kvb_scan."""
import numpy as np
import pytest
import torch

from oracle import gdn_grad
from paper_2605_19049_amd import kvb
from harness import TORCH_DT, UNIT, dev, host, rel_err
from test_gpu_scan import Seqs

pytestmark = pytest.mark.gpu

# Largest error over the RMS.  fp32 gradients: three times the bound of kvb_scan (two passes over the sequence and the
# products that join them, each held to 2^-24).  16-bit gradients: one rounding, and products to 2^-16 of a term, of
# which some ten add up like a random walk.
TOL, TOL16 = 3e-5, 1e-4
SCALE = 0.125


class Grads(Seqs):
    def __init__(self, *args, out_dtype="f32", **kw):
        super().__init__(*args, **kw)
        rng = np.random.default_rng(kw.get("seed", 0) + 1000)
        self.out_dtype = out_dtype
        self.dO = torch.from_numpy(rng.standard_normal((self.N, self.Hv, self.d))).to("cuda").to(TORCH_DT[out_dtype])
        self.dS = (0.1 * rng.standard_normal(self.S.shape)).astype(np.float32)
        self.dstate1 = dev(self.dS)

    def backward(self, state0=True, dstate1=True, dstate0=True, stream=None):
        sh, sq = self.shape(self.out_dtype), self.seqs()
        if self.q.stride(0) > self.Hk * self.d:   # gradients lie as the inputs do
            rows = torch.full((self.N, self.q.stride(0)), 7.0, dtype=self.q.dtype, device="cuda")
            dq, dk, dv = (p.view(self.N, -1, self.d) for p in rows[:, 8:-8].split([self.Hk * self.d, self.Hk * self.d, self.Hv * self.d], dim=1))
        else:
            dq, dk, dv = (torch.full_like(x, 7.0) for x in (self.q, self.k, self.v))
        dg, dbeta, ds0 = torch.full_like(self.g, 7.0), torch.full_like(self.g, 7.0), torch.full_like(self.state0, 7.0)
        work = torch.full((kvb.scan_backward_work(sh, sq) // 4,), float("nan"), device="cuda")
        kvb.kvb_scan_backward(sh, sq, self.q, self.k, self.v, self.g, self.beta, self.state0 if state0 else None, self.dO,
                              self.dstate1 if dstate1 else None, dq, dk, dv, dg, dbeta, ds0 if dstate0 else None, work, stream=stream)
        return dq, dk, dv, dg, dbeta, ds0

    def wanted(self, state0=True, dstate1=True):
        res = [[] for _ in range(6)]
        dO = host(self.dO)
        for b, n in enumerate(self.lens):
            x = [self.x[m][b, :n] for m in ("q", "k", "v", "g", "beta")]
            s = self.slots[b]
            one = gdn_grad.backward(self.S[s] * state0, *x, SCALE, self.unpack(dO, b), self.dS[s] * dstate1)
            for r, y in zip(res, one):
                r.append(y)
        return [np.concatenate(r) for r in res[:5]] + [np.stack(res[5])]

    def check_backward(self, **kw):
        got, want = self.backward(**kw), self.wanted(**{n: y for n, y in kw.items() if n in ("state0", "dstate1")})
        first = self.starts[0]
        errs = {}
        for name, x, y in zip(("dq", "dk", "dv", "dg", "dbeta"), got, want):
            typed = name in ("dq", "dk", "dv") and self.in_dtype != "f32"
            if y.size:
                errs[name] = rel_err(host(x)[first:], y, UNIT[self.in_dtype] if typed else 0.0) / (TOL16 if typed else TOL)
            assert (host(x)[:first] == 7.0).all()
        s0 = host(got[5])
        if kw.get("dstate0", True) and np.sqrt(np.mean(want[5] ** 2)) > 2.0 ** -100:   # (below, 24 bits reach out of fp32's range)
            errs["dstate0"] = rel_err(s0[self.slots], want[5]) / TOL
            assert (s0[np.setdiff1d(np.arange(self.n_slots), self.slots)] == 7.0).all()
        assert max(errs.values()) < 1.0, errs


CASES = [
    # lengths, Hk, Hv, d, inputs, outputs
    ([1], 1, 1, 128, "bf16", "f32"), ([2, 1, 1, 3], 2, 4, 128, "bf16", "bf16"), ([64], 1, 2, 128, "bf16", "f32"),
    ([65, 0, 17, 128], 2, 4, 128, "bf16", "bf16"), ([0, 0, 5], 1, 3, 128, "bf16", "f32"), ([0], 1, 1, 128, "bf16", "f32"),
    ([300, 31, 33], 1, 3, 128, "bf16", "f32"), ([15, 100], 2, 4, 128, "f16", "f16"), ([130, 64], 1, 2, 128, "f16", "f32"),
    ([70, 130, 1], 1, 2, 128, "f32", "f32"), ([70, 130, 1], 3, 9, 64, "bf16", "bf16"), ([191], 2, 4, 64, "f16", "f32"),
    ([100, 257], 1, 2, 64, "f32", "f32"), ([70, 130, 1], 2, 4, 32, "bf16", "f32"), ([17, 99], 2, 2, 32, "f16", "f16"),
    ([100, 64, 63], 1, 2, 32, "f32", "f32"), ([3] * 70 + [130], 1, 1, 32, "bf16", "f32"),
]


@pytest.mark.parametrize("lens, Hk, Hv, d, in_dtype, out_dtype", CASES)
def test_against_the_recurrence(lens, Hk, Hv, d, in_dtype, out_dtype):
    Grads(lens, Hk, Hv, d, in_dtype, seed=len(lens) + d, out_dtype=out_dtype).check_backward()


@pytest.mark.parametrize("in_dtype, d", [("bf16", 128), ("f16", 64), ("f32", 32)])
def test_rows_of_one_projection_and_a_gap_in_front(in_dtype, d):
    Grads([90, 0, 64, 7], 2, 4, d, in_dtype, seed=3, gap=37, fused=True).check_backward()


def test_what_may_be_missing():
    t = Grads([90, 0, 64, 7], 2, 4, 64, "f32", seed=4)
    t.check_backward(state0=False)
    t.check_backward(dstate1=False)
    t.check_backward(dstate0=False)


@pytest.mark.parametrize("g_lo", [0.0, -0.01, -30.0, -1000.0])
def test_decays_of_all_sizes(g_lo):
    Grads([200, 64], 1, 2, 128, "bf16", seed=5, g_lo=g_lo).check_backward()


def test_betas_of_zero_and_one():
    t = Grads([150, 64], 1, 2, 64, "f32", seed=6)
    t.x["beta"][:, ::3] = 0.0
    t.x["beta"][:, 1::3] = 1.0
    t.beta = t.pack(t.x["beta"], False)
    t.check_backward()


@pytest.mark.parametrize("name, at", [("q", 0), ("k", 1), ("v", 2), ("g", 3), ("beta", 4), ("state0", 5)])
def test_against_differences_of_the_forward_pass(name, at):
    """Sums in fp64 of what kvb_scan gives at x + h way and x - h way.  Its outputs are good to 1e-6 of their size, the loss
    is a sum of some thousand of them with random signs: with h = 1e-2 the difference is good to about
    1e-6 sqrt(1e4) / 1e-2 = 1e-2, beside the third derivative's h^2 = 1e-4 of the sum; its size is that of sqrt(1e4) = 100 or more."""
    t = Grads([100, 70], 1, 2, 32, "f32", seed=7)
    grad = t.backward()[at].double()
    gen = torch.Generator(device="cuda").manual_seed(at)
    x = getattr(t, name).clone()
    way = torch.randn(x.shape, generator=gen, device="cuda") * (0.05 if name in ("q", "k", "g", "beta") else 1.0)
    real = torch.zeros(t.n_slots, dtype=torch.bool, device="cuda")
    real[t.slot.long()] = True

    def loss():
        out, s1 = t.scan()
        return float((out.double() * t.dO.double()).sum() + (s1.double() * t.dstate1.double())[real].sum())

    ends = []
    for h in (1e-2, -1e-2):
        setattr(t, name, x + h * way)
        ends.append(loss())
    want = (ends[0] - ends[1]) / 2e-2
    got = float((grad * way.double())[real if name == "state0" else slice(None)].sum())
    assert abs(got - want) < 2e-2 * max(1.0, abs(want)) + 2e-2


def test_same_bits_every_time_and_on_another_stream():
    t = Grads([90, 0, 640, 7], 2, 4, 128, "bf16", seed=8, out_dtype="bf16")
    one = t.backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two = t.backward(stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(one, two))


def test_in_place_gradient_of_the_states():
    t = Grads([90, 64], 1, 2, 64, "bf16", seed=9)
    want = t.backward()[5]
    sh, sq = t.shape(), t.seqs()
    work = torch.empty(kvb.scan_backward_work(sh, sq), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(x) for x in (t.q, t.k, t.v, t.g, t.g)]
    both = t.dstate1.clone()
    kvb.kvb_scan_backward(sh, sq, t.q, t.k, t.v, t.g, t.beta, t.state0, t.dO, both, *outs, both, work)
    assert torch.equal(both[t.slot.long()], want[t.slot.long()])


def test_skipped_sequences_and_bounds_that_make_no_sense():
    t = Grads([100, 80], 1, 2, 64, "bf16", seed=10)
    ref = t.backward()
    t.start = dev(np.array([-50, 100, 10 ** 6], np.int32))
    assert all(torch.equal(x, y) for x, y in zip(t.backward(), ref))
    t.start, t.slot = dev(t.starts), dev(np.array([t.slots[0], t.n_slots], np.int32))
    got = t.backward()
    for x, y in zip(got[:5], ref):
        assert torch.equal(x[:100], y[:100]) and (host(x)[100:] == 7.0).all()


def test_replayed_from_a_graph():
    t = Grads([90, 0, 64, 7], 2, 4, 128, "bf16", seed=11)
    sh, sq = t.shape(), t.seqs()
    outs = [torch.zeros_like(x) for x in (t.q, t.k, t.v, t.g, t.g, t.state0)]
    work = torch.empty(kvb.scan_backward_work(sh, sq), dtype=torch.uint8, device="cuda")

    def call():
        kvb.kvb_scan_backward(sh, sq, t.q, t.k, t.v, t.g, t.beta, t.state0, t.dO, t.dstate1, *outs, work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        t.v.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = t.backward()
        assert all(torch.equal(x, y) for x, y in zip(outs[:5], want[:5])) and torch.equal(outs[5][t.slots], want[5][t.slots])
