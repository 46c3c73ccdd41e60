"""kvb_scan on either side of where its ways part: token by token up to four tokens a sequence, one launch for about a chunk a sequence,
workgroups of four waves or eight.  Bounds and inputs are those of the tests of whole sequences."""
import numpy as np
import pytest
import torch

from paper_2605_19049_amd import kvb
from harness import dev, host, rel_err
from test_gpu_scan import TOL, Seqs

pytestmark = pytest.mark.gpu

CASES = [
    # lengths, Hk, Hv, d, inputs, outputs
    ([1] * 16, 2, 4, 128, "bf16", "bf16"), ([1, 0, 1, 1], 1, 3, 128, "f16", "f32"), ([1, 1], 2, 4, 64, "f32", "f32"),
    ([1] * 70, 1, 2, 32, "bf16", "f32"), ([1, 2], 2, 2, 32, "f16", "f16"), ([1, 1, 0], 1, 2, 128, "f32", "f32"),
    ([16, 0, 0, 0], 2, 4, 128, "bf16", "f32"), ([0, 12, 0, 4], 2, 4, 64, "f16", "f16"), ([0, 0, 0, 14], 1, 2, 32, "f32", "f32"),
    ([4, 4], 2, 4, 128, "bf16", "f32"), ([5, 4], 2, 4, 128, "bf16", "f32"), ([5, 4], 1, 2, 64, "f32", "f32"),
    ([0] * 99 + [300], 1, 1, 64, "bf16", "f32"),                             # one long sequence among many empty ones
    ([37], 2, 4, 128, "bf16", "bf16"), ([64], 1, 2, 128, "f16", "f32"), ([64, 64], 1, 2, 64, "f32", "f32"),
    ([128, 0, 0], 2, 4, 128, "bf16", "f32"), ([0, 190, 2], 2, 4, 128, "f16", "f16"), ([150, 0, 0], 1, 3, 64, "bf16", "bf16"),
    ([64, 65], 2, 4, 128, "bf16", "f32"), ([40] * 33, 2, 4, 128, "bf16", "f32"), ([10] * 65, 1, 2, 64, "f16", "f32"),
    ([70] * 32, 2, 4, 128, "bf16", "bf16"), ([70] * 33, 2, 4, 128, "bf16", "bf16"),
]


@pytest.mark.parametrize("lens, Hk, Hv, d, in_dtype, out_dtype", CASES)
def test_against_the_recurrence(lens, Hk, Hv, d, in_dtype, out_dtype):
    t = Seqs(lens, Hk, Hv, d, in_dtype, seed=sum(lens) + d)
    t.check(*t.scan(out_dtype), *t.expected(), out_dtype)


@pytest.mark.parametrize("lens", [[1, 0, 3, 2], [60, 0, 64, 7]])
@pytest.mark.parametrize("in_dtype, d", [("bf16", 128), ("f16", 64), ("f32", 64)])
def test_strides_a_gap_in_front_no_first_state_and_in_place(lens, in_dtype, d):
    t = Seqs(lens, 2, 4, d, in_dtype, seed=3, gap=3, fused=True)
    t.check(*t.scan(), *t.expected())
    t.check(*t.scan(state0=False), *t.expected(state0=False))
    o, S = t.expected()
    t.state0 = t.state0.clone()
    out, s1 = t.scan(state1=t.state0)
    assert rel_err(host(s1)[t.slots], S) < TOL and rel_err(host(out)[3:], np.concatenate([o[b, :n] for b, n in enumerate(t.lens)])) < TOL


@pytest.mark.parametrize("lens", [[8, 0, 3, 2], [64, 40]])
@pytest.mark.parametrize("g_lo", [0.0, -30.0, -1000.0])
def test_decays_of_all_sizes(lens, g_lo):
    t = Seqs(lens, 1, 2, 128, "bf16", seed=5, g_lo=g_lo)
    t.check(*t.scan(), *t.expected())


@pytest.mark.parametrize("lens", [[8, 0, 2, 3], [60, 0, 64, 50]])
def test_skipped_sequences_and_bounds_that_make_no_sense(lens):
    t = Seqs(lens, 1, 2, 64, "bf16", seed=6)
    out, _ = t.scan()
    n = t.N
    t.start = dev(np.array([-5, lens[0], lens[0], lens[0] + lens[2], 10 ** 6], np.int32))
    again, _ = t.scan()
    assert torch.equal(out, again)
    slots = t.slots.copy()
    t.slot = dev(np.array([slots[0], -1, t.n_slots, slots[3]], np.int32))
    some, s1 = t.scan()
    assert torch.equal(some[:lens[0]], out[:lens[0]]) and torch.equal(some[n - lens[3]:], out[n - lens[3]:])
    assert (some[lens[0]:lens[0] + lens[2]] == 7.0).all() and (host(s1)[slots[1:3]] == 7.0).all()


def test_replayed_from_a_graph():
    for lens in ([1] * 9, [60, 30]):
        t = Seqs(lens, 2, 4, 128, "bf16", seed=7)
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
            got = out.clone(), s1.clone()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got[0], out) and torch.equal(got[1][t.slot.long()], s1[t.slot.long()])
