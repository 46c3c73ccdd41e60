"""kvb_conv and kvb_conv_backward with bounds of sequences that do not ascend: what they give is not said, but nothing outside is touched."""
import pytest
import torch

from paper_2605_19049_amd import kvb
from test_gpu_conv import FILL, Case
from test_gpu_conv_backward import grads_of

pytestmark = pytest.mark.gpu
DESCENDING = [[0, 50, 20, 60], [-5, 50, 20, 1000], [60, 40, 20, 0], [2 ** 31 - 1, -2 ** 31, 7, 3]]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bounds", DESCENDING, ids=str)
def test_results(bounds, dtype):
    """Inside the tokens, and the sequences' own rows of the states"""
    n = 60   # (the arrays have four rows more)
    c = Case([10, 20, 30], 1, 2, 128, 4, dtype, n_slots=5, tail=4)
    c.slot = torch.tensor([0, 3, 1], dtype=torch.int32, device="cuda")
    start = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    sq = kvb.seqs(start, n, c.n_slots, slot=c.slot)
    o, s1, before = c.outs(), torch.full_like(c.state0, FILL), [y.clone() for y in (c.x, c.a, c.b, c.state0)]
    kvb.kvb_conv(c.sh, c.ta, sq, c.x, c.a, c.b, c.state0, s1, *o)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(before, (c.x, c.a, c.b, c.state0)))
    for y in o:
        assert (y[n:] == FILL).all()
    assert (s1[[2, 4]] == FILL).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bounds", DESCENDING, ids=str)
def test_gradients(bounds, dtype):
    """And inside the workspace"""
    n = 60
    c = Case([10, 20, 30], 1, 2, 128, 4, dtype, n_slots=5, tail=4)
    c.slot = torch.tensor([0, 3, 1], dtype=torch.int32, device="cuda")
    c.start = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    g, dx, da, db, ds0 = grads_of(c), *(torch.full_like(y, FILL) for y in (c.x, c.a, c.b, c.state0))
    sq = kvb.seqs(c.start, n, c.n_slots, slot=c.slot)
    room = kvb.conv_backward_work(c.sh, c.ta, sq)
    work = torch.full((room + 65536,), 119, dtype=torch.uint8, device="cuda")
    sums = [torch.empty(c.C, c.W, device="cuda"), None, torch.empty(c.Hv, device="cuda"), torch.empty(c.Hv, device="cuda")]
    kvb.kvb_conv_backward(c.sh, c.ta, sq, c.x, c.a, c.b, c.state0, *g.values(), dx, da, db, *sums, ds0, work)
    torch.cuda.synchronize()
    for y in (dx, da, db):
        assert (y[n:] == FILL).all()
    assert (ds0[[2, 4]] == FILL).all() and (work[room:] == 119).all()
