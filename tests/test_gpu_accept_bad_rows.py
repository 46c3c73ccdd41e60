"""kvb_accept on rows that are no probabilities: what is not a number, and rows that sum to more than fp64 adds up exactly."""
import numpy as np
import pytest
import torch

from accept_reference import accept
from paper_2605_19049_amd import kvb
from harness import dev

pytestmark = pytest.mark.gpu
NAN = np.float32(np.nan)


def run(target, draft, tokens, u, s, parent=None):
    """One request among copies of itself, so that its row is split (one request) or not; (path, accepted, token)."""
    T, V = len(tokens), target.shape[-1]
    res = []
    for B in (1, 200):
        vo = kvb.vocab(B, T, V, kvb.F32)
        many = lambda x: None if x is None else dev(np.ascontiguousarray(np.broadcast_to(np.asarray(x), (B,) + np.shape(x))))
        path = torch.full((B, T), 99, dtype=torch.int32, device="cuda")
        accepted, token = (torch.full((B,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        work = torch.empty(kvb.accept_work(vo), dtype=torch.uint8, device="cuda")
        kvb.kvb_accept(vo, None, many(None if parent is None else np.int32(parent)), many(np.int32(tokens)), many(target), many(draft),
                       many(np.float32(u)), many(np.float32(s)), path, accepted, token, work)
        res.append([x.cpu().numpy() for x in (path, accepted, token)])
        for x in res[-1]:
            assert (x == x[0]).all()
    for x, y in zip(*res):
        assert (x[0] == y[0]).all()
    return res[0][0][0].tolist(), int(res[0][1][0]), int(res[0][2][0])


@pytest.mark.parametrize("V", [64, 40000])
def test_a_chosen_draft_whose_probability_is_not_a_number(V):
    """It counts as 0: the draft is rejected and what is left stays as it was, so that its sibling is accepted as from the whole row."""
    target = np.zeros((3, V), np.float32)
    target[0, [3, 5, 7]] = NAN, 0.25, 0.75
    target[2, 9] = 1.0
    for u, want in ((0.2, ([1, -1], 1, 9)), (0.3, ([-1, -1], 0, 7))):
        got = run(target, None, [3, 5], [0.5, u], 0.1, parent=[-1, -1])
        assert got == want
        target0 = np.nan_to_num(target)
        ref = accept(2, np.array([-1, -1]), np.array([3, 5]), target0, None, np.float32([0.5, u]), np.float32(0.1))
        assert (ref[0].tolist(), ref[1], ref[2]) == want


@pytest.mark.parametrize("V", [64, 40000])
def test_a_drawn_draft_whose_probability_is_not_a_number(V):
    """In a draft's row it counts as infinity: the draft is not accepted, and nothing is left of the token."""
    target, draft = np.zeros((3, V), np.float32), np.zeros((2, V), np.float32)
    target[0, [3, 5, 7]] = 0.5, 0.25, 0.25
    target[2, 9] = 1.0
    draft[0, [3, 5, 7]] = NAN, NAN, 0.125
    draft[1, 7] = 1.0
    for u in (0.0, 0.5):
        # what is left is 0.125 of token 7: drawn at the end of a chain, and more than 0.999 times itself for a sibling
        assert run(target, draft, [3, 7], [u, 0.999], 0.5) == ([-1, -1], 0, 7)
        assert run(target, draft, [3, 7], [u, 0.999], 0.5, [-1, -1]) == ([1, -1], 1, 9)


def test_a_target_row_of_nothing_but_nan():
    for V in (64, 40000):
        assert run(np.full((2, V), NAN), None, [0], [0.0], 0.5) == ([-1], 0, -1)


@pytest.mark.parametrize("V, at", [(600, 0), (600, 290), (40000, 0), (40000, 20000), (70000, 65400)])
def test_a_row_that_sums_to_more_than_fp64_holds_exactly(V, at):
    """100 ones, 100 values of 2^-48, 100 ones: with s = 1/2 the running sums that lie on either side of the aim differ by less than
    their rounding.  A token of the row comes out all the same, one of those next to the aim."""
    target = np.zeros((2, V), np.float32)
    target[0, at:at + 300] = 1.0
    target[0, at + 100:at + 200] = 2.0 ** -48
    path, accepted, token = run(target, None, [V - 1], [0.5], 0.5)
    assert path == [-1] and accepted == 0 and at + 99 <= token <= at + 200
