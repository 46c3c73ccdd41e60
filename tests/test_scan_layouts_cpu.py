"""Tensors that do not lie as a scan's kvb_seqs says are refused by the binding (no GPU: calls of no sequences, which launch nothing)."""
import pytest
import torch

from paper_2605_19049_amd import kvb

N, Hk, Hv, D = 10, 2, 4, 64
SH = kvb.shape(0, Hk, Hv, D, D, 1, kvb.F32)
NAMES = ("q", "k", "v", "g", "beta", "state0", "dout", "dstate1", "dq", "dk", "dv", "dg", "dbeta", "dstate0")


def projection(n=N):
    """q, k and v as parts of the rows of one projection."""
    return [x.view(n, -1, D) for x in torch.zeros(n, (2 * Hk + Hv) * D).split([Hk * D, Hk * D, Hv * D], dim=1)]


def packed(n=N):
    return [torch.zeros(n, h, D) for h in (Hk, Hk, Hv)]


def arrays(rows, grads, n=N):
    a = dict(zip("qkv", rows))
    a.update(zip(("dq", "dk", "dv"), grads))
    a.update({x: torch.zeros(n, Hv) for x in ("g", "beta", "dg", "dbeta")})
    a.update({x: torch.zeros(1, Hv, D, D) for x in ("state0", "dstate1", "dstate0")})
    a["dout"] = torch.zeros(n, Hv, D)
    return a


def backward(a, sq, bound):
    args = [SH, sq] + [a[x] for x in NAMES] + [torch.zeros(64)]
    if bound:
        return kvb.bind("kvb_scan_backward", *args, 0)()
    return kvb.kvb_scan_backward(*args, stream=0)


def forward(a, sq, bound):
    args = [SH, sq] + [a[x] for x in NAMES[:6]] + [a["state0"], a.get("out", a["dout"]), torch.zeros(64)]
    if bound:
        return kvb.bind("kvb_scan", *args, 0)()
    return kvb.kvb_scan(*args, stream=0)


def seqs(rows, n=N):
    return kvb.seqs(torch.zeros(1, dtype=torch.int32), n, 1, **dict(zip("qkv", rows)))


@pytest.mark.parametrize("bound", [False, True])
def test_gradients_lie_as_their_inputs_do(bound):
    q, k, v = projection()
    sq = seqs((q, k, v))
    assert sq.q_stride == (2 * Hk + Hv) * D
    backward(arrays((q, k, v), projection()), sq, bound)
    for i in range(3):   # (empty_like of a part of a row is packed: rows of the projection apart, its end would be written behind)
        grads = projection()
        grads[i] = torch.empty_like((q, k, v)[i])
        with pytest.raises(ValueError):
            backward(arrays((q, k, v), grads), sq, bound)
    backward(arrays(packed(), packed()), seqs(packed()), bound)
    backward(arrays(packed(), packed()), seqs([]), bound)
    with pytest.raises(ValueError):
        backward(arrays(packed(), projection()), seqs(packed()), bound)


@pytest.mark.parametrize("bound", [False, True])
@pytest.mark.parametrize("call", [forward, backward])
def test_inputs_lie_as_their_sequences_say(call, bound):
    for rows, said in ((projection(), packed()), (packed(), projection()), (projection(), [])):
        with pytest.raises(ValueError):
            call(arrays(rows, said or packed()), seqs(said), bound)
    call(arrays(projection(), projection()), seqs(projection()), bound)
    with pytest.raises(ValueError):   # heads that do not follow each other
        call(arrays([x.transpose(0, 1).contiguous().transpose(0, 1) for x in packed()], packed()), seqs(packed()), bound)


@pytest.mark.parametrize("bound", [False, True])
def test_rows_without_heads_and_addresses(bound):
    flat = [x.view(N, -1) for x in packed()]
    backward(arrays(flat, flat), seqs([]), bound)
    parts = [x.flatten(1) if x.is_contiguous() else x.as_strided((N, x.shape[1] * D), (x.stride(0), 1)) for x in projection()]
    backward(arrays(parts, parts), seqs(projection()), bound)
    with pytest.raises(ValueError):
        backward(arrays(parts, flat), seqs(projection()), bound)
    backward({x: 4096 for x in NAMES}, seqs(projection()), bound)


@pytest.mark.parametrize("n", [1, 2])
def test_heads_of_a_single_token_follow_each_other(n):
    """A part of each head's row: heads 3 d apart, which no stride of a kvb_seqs says."""
    x = torch.zeros(n, Hk, 3 * D)[:, :, :D]
    for bad in (x, torch.zeros(n, Hk, 2 * D)[:, :, ::2], torch.zeros(n, Hk, 1).expand(n, Hk, D), torch.zeros(D, Hk, n).permute(2, 1, 0)):
        with pytest.raises(ValueError):
            kvb.seqs(0, n, 1, q=bad)
        with pytest.raises(ValueError):
            forward(arrays([bad] + packed(n)[1:], packed(n), n), seqs([], n), False)
    assert kvb.seqs(0, n, 1, q=torch.zeros(n, 1, 3 * D)[:, :, :D]).q_stride == (0 if n == 1 else 3 * D)   # (one head: rows apart)
    assert kvb.seqs(0, 0, 1, q=torch.zeros(0, Hk, D)).q_stride == 0


@pytest.mark.parametrize("bound", [False, True])
def test_what_has_no_stride_is_packed(bound):
    """Gates as columns of a projection's rows, transposed or broadcast gradients: there is no stride that could say so."""
    q, k, v = packed()
    wide = torch.zeros(N, 2 * Hv + 3)
    for name, bad in (("g", wide[:, :Hv]), ("beta", wide[:, Hv:2 * Hv]), ("state0", torch.zeros(1, Hv, D, 2 * D)[..., :D])):
        for call in (forward, backward):
            with pytest.raises(ValueError):
                call({**arrays((q, k, v), packed()), name: bad}, seqs((q, k, v)), bound)
    for name, bad in (("dout", torch.zeros(1, 1, D).expand(N, Hv, D)), ("dg", wide[:, :Hv]), ("dbeta", torch.zeros(Hv, N).t()),
                      ("dstate1", torch.zeros(1, Hv, D, D).transpose(2, 3)), ("dstate0", torch.zeros(1, Hv, D, D).transpose(2, 3))):
        with pytest.raises(ValueError):
            backward({**arrays((q, k, v), packed()), name: bad}, seqs((q, k, v)), bound)
    with pytest.raises(ValueError):
        forward({**arrays((q, k, v), packed()), "out": torch.zeros(Hv, N, D).transpose(0, 1)}, seqs((q, k, v)), bound)
    a = arrays((q, k, v), packed())
    a.update(g=torch.zeros(2 * N, Hv)[N:], state0=None, dstate1=None, dstate0=None)   # (contiguous; not there)
    backward(a, seqs((q, k, v)), bound)
    forward(a, seqs((q, k, v)), bound)
