"""kvb_accept against a plain statement of it, bit for bit: chains and trees, drawn and chosen drafts, rows of all lengths."""
import numpy as np
import pytest
import torch

from accept_reference import accept
from paper_2605_19049_amd import kvb
from harness import DT, TORCH_DT, dev

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, B, T, V, dtype, draft, tree, seed=0, sharp=3.0, pad=0):
        rng = np.random.default_rng(seed)
        self.B, self.T, self.V, self.dtype, self.pad = B, T, V, dtype, pad
        logits = sharp * rng.standard_normal((B, T + 1, V))
        self.target = self.probs(logits)
        self.parent = None
        up = np.broadcast_to(np.arange(T) - 1, (B, T)).copy()
        if tree:
            up = self.parent = np.floor(rng.random((B, T)) * (np.arange(T) + 1)).astype(np.int32) - 1
        bb = np.arange(B)[:, None]
        near = logits[bb, up + 1] + (0.8 * rng.standard_normal((B, T + 1, V)))[bb, up + 1]
        self.draft = self.probs(near) if draft else None
        if draft:
            c = self.draft.astype(np.float64).cumsum(-1)
            self.tokens = np.minimum((c < rng.random((B, T, 1)) * c[..., -1:]).sum(-1), V - 1)
        else:
            order = np.argsort(-near, axis=-1)[..., :T]
            rank = np.array([[sum(up[b, k] == up[b, i] for k in range(i)) for i in range(T)] for b in range(B)])
            self.tokens = np.take_along_axis(order, np.minimum(rank, V - 1)[..., None], -1)[..., 0]
        self.tokens = self.tokens.astype(np.int32)
        self.u, self.s = rng.random((B, T)).astype(np.float32), rng.random(B).astype(np.float32)
        self.u, self.s = np.minimum(self.u, np.float32(1 - 2.0 ** -24)), np.minimum(self.s, np.float32(1 - 2.0 ** -24))
        self.n = None

    def probs(self, x):
        e = np.exp(x - x.max(-1, keepdims=True))
        return torch.from_numpy((e / e.sum(-1, keepdims=True)).astype(np.float32)).to(TORCH_DT[self.dtype]).float().numpy()

    def rows(self, x):
        if x is None:
            return None
        y = torch.full(x.shape[:-1] + (self.V + self.pad,), 0.25, dtype=TORCH_DT[self.dtype], device="cuda")
        y[..., :self.V] = dev(x, self.dtype)
        return y

    def run(self, stream=None):
        vo = kvb.vocab(self.B, self.T, self.V, DT[self.dtype], self.V + self.pad if self.pad else 0)
        work = torch.full((kvb.accept_work(vo) // 8,), float("nan"), dtype=torch.float64, device="cuda")
        path = torch.full((self.B, self.T), 99, dtype=torch.int32, device="cuda")
        accepted, token = (torch.full((self.B,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
        kvb.kvb_accept(vo, None if self.n is None else dev(self.n), None if self.parent is None else dev(self.parent), dev(self.tokens),
                       self.rows(self.target), self.rows(self.draft), dev(self.u), dev(self.s), path, accepted, token, work, stream=stream)
        torch.cuda.synchronize()
        return path.cpu().numpy(), accepted.cpu().numpy(), token.cpu().numpy()

    def check(self):
        path, accepted, token = self.run()
        for b in range(self.B):
            n = self.T if self.n is None else int(min(max(self.n[b], 0), self.T))
            want = accept(n, None if self.parent is None else self.parent[b], self.tokens[b], self.target[b],
                          None if self.draft is None else self.draft[b], self.u[b], self.s[b])
            assert (path[b] == want[0]).all() and accepted[b] == want[1] and token[b] == want[2], (b, path[b], accepted[b], token[b], want)
        return path, accepted, token


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("B, T, V, dtype", [(3, 1, 1, "f32"), (5, 4, 7, "bf16"), (4, 8, 8, "f32"), (6, 5, 511, "f16"), (5, 8, 1000, "f32"),
                                            (2, 3, 4097, "bf16"), (40, 4, 300, "f16"), (1, 8, 33333, "f32"), (3, 2, 50001, "bf16")])
def test_against_the_plain_statement(B, T, V, dtype, draft, tree):
    Case(B, T, V, dtype, draft, tree, seed=B + 10 * T).check()


@pytest.mark.parametrize("draft", [False, True])
def test_rows_split_over_workgroups_or_not(draft):
    """The same request alone (its row in segments) and among so many that a workgroup has a row."""
    one = Case(1, 3, 40000, "f32", draft, False, seed=5)
    want = one.check()
    many = Case(1, 3, 40000, "f32", draft, False, seed=5)
    B = many.B = 600
    for name in ("target", "draft", "tokens", "u", "s"):
        x = getattr(one, name)
        setattr(many, name, None if x is None else np.repeat(x, B, 0))
    assert kvb.accept_work(kvb.vocab(B, 3, 40000, kvb.F32)) == 8 * B < 8 * B * kvb.accept_work(kvb.vocab(1, 3, 40000, kvb.F32)) // 8
    for got, w in zip(many.run(), want):
        assert (got == w[0]).all()


def test_ragged_numbers_of_drafts():
    for tree in (False, True):
        c = Case(9, 6, 700, "f32", True, tree, seed=6)
        c.n = np.array([0, 1, 2, 3, 4, 5, 6, -3, 100], np.int32)
        c.check()


def test_padded_rows():
    for draft, tree, dtype in ((True, False, "bf16"), (True, True, "f32"), (False, True, "f16")):
        Case(4, 4, 1003, dtype, draft, tree, seed=7, pad=13).check()


def test_parents_and_tokens_out_of_range():
    c = Case(4, 6, 100, "f32", True, True, seed=8)
    c.parent[0, 2], c.parent[1, 3], c.parent[2, 1] = 5, -7, 1
    c.tokens[0, 0], c.tokens[1, 1], c.tokens[3, 0] = -1, 100, 2 ** 31 - 1
    c.check()
    c = Case(4, 6, 100, "f32", False, True, seed=8)
    c.tokens[0, 0], c.tokens[1, 1], c.tokens[3, 0] = -1, 100, -2 ** 31
    c.check()


@pytest.mark.parametrize("tree", [False, True])
def test_edges_of_the_probabilities(tree):
    """Rows of zeros, one certain token, target and draft the same (nothing is left), NaN, infinity, random numbers at their ends."""
    c = Case(10, 4, 600, "f32", True, tree, seed=9)
    c.target[0] = 0.0
    c.target[1] = 0.0
    c.target[1, :, 599] = 1.0
    c.target[2] = 0.0
    c.target[2, :, 0] = 1.0
    c.draft[3] = c.target[3, :1]
    c.target[3] = c.target[3, :1]
    c.target[4, :, ::3] = np.nan
    c.draft[5, :, ::3] = np.nan
    c.target[6, :, 7] = np.inf
    c.u[7], c.s[7] = 0.0, 0.0
    c.u[8], c.s[8] = 1 - 2.0 ** -24, 1 - 2.0 ** -24
    c.draft[9] = 1.0   # more than the target everywhere: nothing is left
    c.u[9] = 1 - 2.0 ** -24
    path, accepted, token = c.check()
    assert accepted[0] == 0 and token[0] == -1 and token[2] in (0,) and accepted[9] == 0


def test_tiny_probabilities_and_ties_of_the_aim():
    """Weights that round down to nothing are never drawn, and an aim that equals a running sum takes the next token."""
    c = Case(3, 1, 64, "f32", False, False, seed=10)
    c.n = np.zeros(3, np.int32)
    c.target[:, 0] = 0.0
    c.target[0, 0, 5:9] = 0.25
    c.target[1, 0, 5:9] = 2.0 ** -50
    c.target[1, 0, 20] = 2.0 ** -48
    c.target[2, 0, 63] = 2.0 ** -126
    c.s[:] = [0.5, 0.999, 0.5]
    _, _, token = c.check()
    assert token.tolist() == [7, 20, -1]


@pytest.mark.parametrize("tree", [False, True])
def test_what_comes_out_is_distributed_as_the_target(tree):
    """One draft, or two siblings, drawn from q: over a grid of random numbers the first emitted token has the target's
    probabilities, to what the grid's steps let through (one step of u for each test, one of s)."""
    rng = np.random.default_rng(11)
    V, G = 5, 48
    p, q = rng.dirichlet(np.ones(V)).astype(np.float32), rng.dirichlet(np.ones(V)).astype(np.float32)
    T = 2 if tree else 1
    grid = (np.arange(G) + 0.5) / G
    freq = np.zeros(V)
    for first in range(V):
        for second in range(V if tree else 1):
            mesh = np.meshgrid(*[grid] * (T + 1), indexing="ij")
            c = Case(G ** (T + 1), T, V, "f32", True, tree, seed=12)
            c.target[:], c.draft[:] = p, q
            c.tokens[:] = [first, second][:T]
            c.parent = np.full((c.B, T), -1, np.int32) if tree else None
            c.u, c.s = np.stack([m.ravel() for m in mesh[:T]], 1).astype(np.float32), mesh[T].ravel().astype(np.float32)
            path, accepted, token = c.run()
            out = np.where(accepted > 0, c.tokens[np.arange(c.B), np.maximum(path[:, 0], 0)], token)
            share = q[first] * (q[second] if tree else 1.0)
            freq += share * np.bincount(out, minlength=V) / c.B
    assert np.abs(freq - p).max() < (T + 1) / G


def test_replayed_from_a_graph_and_on_another_stream():
    c = Case(2, 4, 30000, "f32", True, False, seed=13)
    vo = kvb.vocab(c.B, c.T, c.V, kvb.F32)
    work = torch.empty(kvb.accept_work(vo), dtype=torch.uint8, device="cuda")
    path, (accepted, token) = torch.zeros((2, 4), dtype=torch.int32, device="cuda"), torch.zeros((2, 2), dtype=torch.int32, device="cuda")
    args = [dev(c.tokens), c.rows(c.target), c.rows(c.draft), dev(c.u), dev(c.s)]

    def call():
        kvb.kvb_accept(vo, None, None, *args, path, accepted, token, work)

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
