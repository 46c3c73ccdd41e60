"""kvb_accept's edges on rows so long that they are split over workgroups (two launches): what the short rows' tests hold, again."""
import numpy as np
import pytest
import torch

from paper_2605_19049_amd import kvb
from harness import dev
from test_gpu_accept import Case

pytestmark = pytest.mark.gpu
LONG = [33000, 70001, 140000]   # segments of unequal length at the end; the last one with a line of few tokens


@pytest.mark.parametrize("V", LONG)
@pytest.mark.parametrize("draft, tree", [(True, False), (False, True), (False, False), (True, True)])
def test_edges_of_the_probabilities(V, draft, tree):
    """Rows of zeros, one certain token at either end, target and draft the same, NaN, infinity, random numbers at their ends."""
    c = Case(8, 4, V, "f32", draft, tree, seed=9)
    c.target[0] = 0.0                       # no token
    c.target[1] = 0.0
    c.target[1, :, V - 1] = 1.0
    c.target[2] = 0.0
    c.target[2, :, 0] = 1.0
    c.target[4, :, 1::3] = np.nan
    c.target[5, :, 7] = np.inf
    c.u[6], c.s[6] = 0.0, 0.0
    c.u[7], c.s[7] = 1 - 2.0 ** -24, 1 - 2.0 ** -24
    if draft:
        c.draft[2] = 1.0                    # more than the target everywhere: nothing is left, the target's row again
        c.u[2] = 1 - 2.0 ** -24
        c.draft[3] = c.target[3, :1]
        c.target[3] = c.target[3, :1]
    else:
        c.tokens[2], c.u[2] = 0, 1.0        # the only token of the row is rejected: nothing is left, the target's row again
        c.tokens[4] -= c.tokens[4] % 3 == 1   # (the plain statement's Z is NaN behind a chosen draft without a number)
        c.tokens[4] = np.maximum(c.tokens[4], 0)
    path, accepted, token = c.check()
    assert accepted[0] == 0 and token[0] == -1 and accepted[2] == 0 and token[2] == 0
    if accepted[1] == 0:
        assert token[1] == V - 1


@pytest.mark.parametrize("tree", [False, True])
def test_ragged_numbers_of_drafts_and_padded_rows(tree):
    c = Case(6, 4, 40001, "bf16", not tree, tree, seed=6, pad=7)
    c.n = np.array([0, 1, 2, 3, 4, -3], np.int32)
    c.check()


@pytest.mark.parametrize("tree", [False, True])
def test_replayed_from_a_graph_and_on_another_stream(tree):
    c = Case(2, 4, 40000, "f32", not tree, tree, seed=13)
    vo = kvb.vocab(c.B, c.T, c.V, kvb.F32)
    work = torch.empty(kvb.accept_work(vo), dtype=torch.uint8, device="cuda")
    path, (accepted, token) = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    parent = dev(c.parent) if tree else None
    args = [dev(c.tokens), c.rows(c.target), c.rows(c.draft), dev(c.u), dev(c.s)]

    def call():
        kvb.kvb_accept(vo, None, parent, *args, path, accepted, token, work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    rng = np.random.default_rng(1)
    for _ in range(3):
        c.u, c.s = rng.random((2, 4)).astype(np.float32) * 0.99, rng.random(2).astype(np.float32) * 0.99
        args[3].copy_(dev(c.u)), args[4].copy_(dev(c.s))
        graph.replay()
        torch.cuda.synchronize()
        want = c.check()
        assert (path.cpu().numpy() == want[0]).all() and (accepted.cpu().numpy() == want[1]).all() and (token.cpu().numpy() == want[2]).all()


def test_one_workspace_for_batches_of_all_sizes():
    """Sized for 200 requests, whose rows are not split, it serves fewer, whose rows are; nothing is written behind it."""
    V = 150001
    size = kvb.accept_work(kvb.vocab(200, 2, V, kvb.BF16))
    room = torch.full((size // 8 + 4096,), 7.0, dtype=torch.float64, device="cuda")
    for B in (1, 40, 64, 65, 128, 129, 200):
        c = Case(1, 2, V, "bf16", False, False, seed=B)
        want = c.check()
        many = lambda x: dev(np.repeat(x, B, 0))
        path, (accepted, token) = torch.zeros((B, 2), dtype=torch.int32, device="cuda"), torch.zeros((2, B), dtype=torch.int32, device="cuda")
        target = c.rows(c.target).expand(B, 3, V).contiguous()
        kvb.kvb_accept(kvb.vocab(B, 2, V, kvb.BF16), None, None, many(c.tokens), target, None, many(c.u), many(c.s), path, accepted, token, room)
        torch.cuda.synchronize()
        assert all((x.cpu().numpy() == w[0]).all() for x, w in zip((path, accepted, token), want))
        assert (room[size // 8:] == 7.0).all()
