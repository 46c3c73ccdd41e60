"""kvb_conv_backward against the formulas in 64 bits, and against differences."""
import pytest
import torch

from paper_2605_19049_amd import kvb
from layer_reference import V, f64, gates, softplus, zeros
from running_error import U, check
from test_gpu_conv import EPS, FILL, Case, run

pytestmark = pytest.mark.gpu


def grads_of(c, seed=1, gated=True):
    gen = torch.Generator().manual_seed(seed)
    d = {"d" + n: torch.randn(c.N, h, c.d, generator=gen).to(c.dt).cuda() for n, h in (("q", c.Hk), ("k", c.Hk), ("v", c.Hv))}
    d["dg"], d["dbeta"] = (torch.randn(c.N, c.Hv, generator=gen).cuda() if gated else None for _ in range(2))
    d["dstate1"] = torch.randn(c.state0.shape, generator=gen).to(c.dt).cuda()
    return d


def backward(c, d, state0=True, dstate1=True, dstate0=True, gated=True, fused=False, unit=True, stream=None, work=None):
    if fused:
        row = torch.full((c.N, c.x.stride(0)), FILL, dtype=c.dt, device="cuda")
        dx, da, db = row[:, :c.C], row[:, c.C + 24:][:, :c.Hv], row[:, c.C + 24:][:, c.Hv:2 * c.Hv]
    else:
        dx, da, db = (torch.full_like(y, FILL) for y in (c.x, c.a, c.b))
    r = {"dx": dx, "da": da if gated else None, "db": db if gated else None, "dweight": torch.empty(c.C, c.W, device="cuda"),
         "dbias": torch.empty(c.C, device="cuda") if c.bias is not None else None, "dA_log": torch.empty(c.Hv, device="cuda") if gated else None,
         "ddt_bias": torch.empty(c.Hv, device="cuda") if gated else None, "dstate0": torch.full_like(c.state0, FILL) if dstate0 else None}
    sq, ta = kvb.seqs(c.start, c.N, c.n_slots, slot=c.slot, q=d["dq"], k=d["dk"], v=d["dv"]), c.taps(unit)
    work = torch.empty(kvb.conv_backward_work(c.sh, ta, sq), dtype=torch.uint8, device="cuda") if work is None else work
    kvb.kvb_conv_backward(c.sh, ta, sq, c.x, *((c.a, c.b) if gated else (None, None)), c.state0 if state0 else None, d["dq"], d["dk"], d["dv"], d["dg"],
                          d["dbeta"], d["dstate1"] if dstate1 else None, *r.values(), work, stream=stream)
    torch.cuda.synchronize()
    return r


def check_backward(c, d, r, state0=True, dstate1=True, gated=True, skipped=(), unit=True):
    dw, dbias = zeros(c.C, c.W), zeros(c.C)
    touched, slots = torch.zeros(c.N, dtype=torch.bool), set()
    for b, n in enumerate(c.lens):
        if b in skipped:
            continue
        row, at = int(c.slot[b]), slice(c.ends[b], c.ends[b + 1])
        slots.add(row)
        touched[at] = True
        conv = c.conv_of(c.state0[row] if state0 else None, at, unit)
        dn = f64(torch.cat([d["dq"][at], d["dk"][at], d["dv"][at]], 1))
        dE = conv.backward(dn, f64(d["dstate1"][row]) if dstate1 else None)
        if n:
            check(r["dx"][at], dE[c.W - 1:], "dx")
        if r["dstate0"] is not None:
            check(r["dstate0"][row], dE[:c.W - 1], "dstate0")
        # (a term is added to a sum of at most 32 before it; the sums of waves, workgroups and parts are few)
        for i in range(c.W):
            t = (conv.dz * conv.E[i:i + n]).sum(0, 64, keepdim=False)
            dw.v[:, i] += t.v
            dw.e[:, i] += t.e
        t = conv.dz.sum(0, 64, keepdim=False)
        dbias = V(dbias.v + t.v, dbias.e + t.e)
    check(r["dweight"], dw, "dweight")
    if c.bias is not None:
        check(r["dbias"], dbias, "dbias")
    assert (r["dx"][~touched] == FILL).all()
    if gated:
        at = touched.nonzero()[:, 0]
        rate, y, beta = gates(c.a[at], c.b[at], c.A_log, c.dt_bias)
        dg, dbeta = f64(d["dg"][at]), f64(d["dbeta"][at])
        s = torch.sigmoid(y.v)
        s = V(s, s * (1.0 - s) * (y.e + 4.0) + 3.0 * s)
        da = dg * rate * s
        other = V(1.0 - beta.v, beta.e * 0 + (1.0 - beta.v) * (beta.v * 8.0 + 4.0))
        check(r["da"][at], da, "da")
        check(r["db"][at], dbeta * (beta * other), "db")
        check(r["dA_log"], (dg * (rate * softplus(y))).sum(0, 64 + len(at) // 16, keepdim=False), "dA_log")
        check(r["ddt_bias"], da.sum(0, 64 + len(at) // 16, keepdim=False), "ddt_bias")
        assert (r["da"][~touched] == FILL).all() and (r["db"][~touched] == FILL).all()
    if r["dstate0"] is not None:
        for row in set(range(c.n_slots)) - slots:
            assert (r["dstate0"][row] == FILL).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lens", [[1], [5], [1, 2, 3, 4, 0, 7], [33, 0, 64, 65, 1, 32, 31], [300], [0, 0, 2]], ids=str)
@pytest.mark.parametrize("W, heads, d", [(4, (2, 4), 128), (3, (3, 9), 64), (2, (1, 1), 32), (4, (5, 5), 32)])
def test_gradients(lens, W, heads, d, dtype):
    c = Case(lens, *heads, d, W, dtype, seed=len(lens), bias=W != 4)
    g = grads_of(c)
    check_backward(c, g, backward(c, g))


def test_rows_of_one_projection_rows_of_nobody_and_skipped_ones():
    c = Case([40, 3, 0, 17], 2, 4, 128, 4, "bf16", fused=True, n_slots=9, lead=5, tail=11)
    g = grads_of(c)
    check_backward(c, g, backward(c, g, fused=True))
    c.slot[1] = -3
    check_backward(c, g, backward(c, g, fused=True), skipped=(1,))


def test_without_states_gates_unit():
    c = Case([20, 2, 0, 50], 2, 4, 64, 4, "f32", seed=2, bias=True)
    g = grads_of(c, gated=False)
    check_backward(c, g, backward(c, g, state0=False, dstate1=False, gated=False, dstate0=False), state0=False, dstate1=False, gated=False)
    check_backward(c, g, backward(c, g, dstate1=False, gated=False, unit=False), dstate1=False, gated=False, unit=False)


def test_many_heads():
    """More heads than a wave has lanes"""
    c = Case([40], 35, 70, 32, 4, "f32", seed=3)
    g = grads_of(c)
    check_backward(c, g, backward(c, g))
    o, _ = run(c)
    c.check_gates(o, slice(0, 40))


def test_no_tokens():
    """Sums over nothing are zero; an empty sequence's first state gets its last one's gradient"""
    c = Case([0, 0], 2, 4, 64, 4, "bf16", bias=True)
    g = grads_of(c)
    r = backward(c, g)
    assert all((r[n] == 0).all() for n in ("dweight", "dbias", "dA_log", "ddt_bias"))
    assert torch.equal(r["dstate0"], g["dstate1"])
    c.sh.B = 0
    r = backward(c, g)
    assert all((r[n] == 0).all() for n in ("dweight", "dbias", "dA_log", "ddt_bias"))


def test_tokens_of_nobody():
    c = Case([5, 8], 1, 2, 32, 3, "f32", bias=True)
    d = grads_of(c)
    c.sh, c.start = kvb.shape(0, c.Hk, c.Hv, c.d, c.d, 1, kvb.F32), c.start[:1]
    r = backward(c, d)
    for name in ("dweight", "dbias", "dA_log", "ddt_bias"):
        assert (r[name] == 0).all(), name
    for name in ("dx", "da", "db", "dstate0"):
        assert (r[name] == FILL).all(), name


def test_a_wave_takes_several_short_sequences():
    """More sequences than waves: 300, 224 waves for each 512 channels"""
    c = Case([(b * 5 + b // 7) % 5 for b in range(300)], 8, 16, 128, 4, "bf16", seed=7, bias=True)
    g = grads_of(c)
    check_backward(c, g, backward(c, g))


def test_parts_of_sequences():
    """Waves that have the end of a sequence, whole ones, empty ones and the beginning of another, rows of nobody ahead and behind"""
    c = Case([(b * 11 + b // 5) % 31 * (b % 4 != 2) for b in range(130)], 3, 6, 64, 3, "f32", seed=11, bias=True, n_slots=140, lead=9, tail=4)
    c.slot[17], c.slot[60] = -1, 140
    g = grads_of(c)
    check_backward(c, g, backward(c, g), skipped=(17, 60))


def sum_of_sizes(c, g):
    """sum over tokens of |dz E| for each weight, in 64 bits"""
    lens = (c.start[1:] - c.start[:-1]).long().cpu()
    first, slot = c.start[:-1].long().cpu().repeat_interleave(lens), c.slot.long().cpu().repeat_interleave(lens)
    token = torch.arange(int(c.start[0]), int(c.start[-1]))
    x, state, w = (y.double().cpu() for y in (c.x, c.state0, c.weight))
    E = []
    for i in range(c.W):
        at = token - first + i   # the row of E
        E.append(torch.where((at >= c.W - 1)[:, None], x[(token + i - (c.W - 1)).clamp(min=0)], state[slot, at.clamp(max=c.W - 2)]))
    z = sum(w[:, i] * E[i] for i in range(c.W)).requires_grad_()
    y = z * torch.sigmoid(z)
    h = y.unflatten(1, (-1, c.d))
    n = torch.cat([h[:, :2 * c.Hk] / (h[:, :2 * c.Hk].square().sum(-1, keepdim=True) + EPS).sqrt(), h[:, 2 * c.Hk:]], 1)
    dn = torch.cat([g[k][token] for k in ("dq", "dk", "dv")], 1).double().cpu()
    (dz,) = torch.autograd.grad((n * dn).sum(), z)
    return torch.stack([(dz * e).abs().sum(0) for e in E], 1)


@pytest.mark.parametrize("B", [64, 65, 4096, 4097, 6000])
def test_many_sequences(B):
    """Found among up to thousands, two of three empty: token by token the bits of the call that has the others alone"""
    lens = [0 if b % 3 else 1 + b % 4 for b in range(B)]
    c = Case(lens, 1, 2, 32, 4, "f32", seed=B)
    g = grads_of(c)
    r = backward(c, g)
    some = torch.tensor([n > 0 for n in lens], device="cuda")
    none = c.slot[~some].long()
    assert torch.equal(r["dstate0"][none], g["dstate1"][none])
    c.slot, c.start = c.slot[some].contiguous(), torch.cat([c.start[:1], c.start[1:][some]])
    c.sh = kvb.shape(len(c.slot), 1, 2, 32, 32, 1, c.code)
    alone = backward(c, g)
    for n in ("dx", "da", "db"):
        assert torch.equal(r[n], alone[n]), n
    slots = c.slot.long()
    assert torch.equal(r["dstate0"][slots], alone["dstate0"][slots])
    # both are sums of the same numbers dz E: up to 40 tokens a wave, 4 waves, up to 384 parts as 64 sums of 6 each, so fewer than 128 roundings of what their sizes add up to
    size = sum_of_sizes(c, g)
    assert ((r["dweight"] - alone["dweight"]).abs().double().cpu() <= 2 * 128 * U * size).all()


def test_long_sequences():
    """Pieces of some forty tokens; the sums over tokens"""
    c = Case([20001, 20000], 1, 1, 32, 4, "bf16", seed=4)
    g = grads_of(c)
    whole = backward(c, g)
    conv = c.conv_of(c.state0[int(c.slot[1])], slice(20001, 20001 + 300))
    dE = conv.backward(f64(torch.cat([g[n][20001:20301] for n in ("dq", "dk", "dv")], 1)), None)
    check(whole["dx"][20001:20001 + 290], dE[c.W - 1:c.W - 1 + 290], "dx")
    check(whole["dstate0"][int(c.slot[1])], dE[:c.W - 1], "dstate0")
    want = torch.zeros(c.C, c.W, dtype=torch.float64)
    size = torch.zeros(c.C, c.W, dtype=torch.float64)
    worst = torch.zeros(c.C, c.W, dtype=torch.float64)
    for b in range(2):
        conv = c.conv_of(c.state0[int(c.slot[b])], slice(c.ends[b], c.ends[b + 1]))
        conv.backward(f64(torch.cat([g[n][c.ends[b]:c.ends[b + 1]] for n in ("dq", "dk", "dv")], 1)), None)
        for i in range(c.W):
            t = conv.dz * conv.E[i:i + conv.n]
            want[:, i] += t.v.sum(0)
            size[:, i] += t.v.abs().sum(0)
            worst[:, i] += t.e.sum(0)
    # a piece a wave, four waves, up to 256 parts in 16 sums or 64
    check(whole["dweight"], V(want, worst + (64 + 4 + 16 + 64) * size), "dweight")


def test_zero_rows_with_the_least_eps():
    """Rows of zeros have keys of zero; what reaches them is the gradient over sqrt(eps), and nothing that is not a number"""
    c = Case([20], 1, 2, 64, 4, "f32", seed=9)
    c.x.zero_()
    c.state0.zero_()
    g = grads_of(c)
    c.ta = kvb.taps(c.weight, width=4, A_log=c.A_log, dt_bias=c.dt_bias, eps=kvb.MIN_EPS)
    c.taps = lambda unit=True: c.ta
    r = backward(c, g)
    assert all(torch.isfinite(y).all() for y in r.values() if y is not None)
    dz = 0.5 * g["dk"].double().flatten(1) * 1e15   # silu's slope at 0, 1 / sqrt(1e-30)
    w = c.weight[64:128].double()
    want = sum(w[:, i] * torch.nn.functional.pad(dz, (0, 0, 0, 3))[3 - i:23 - i] for i in range(4))
    assert ((r["dx"][:, 64:128].double() - want).abs() <= 32 * 2.0 ** -24 * sum(w[:, i].abs() * torch.nn.functional.pad(dz.abs(), (0, 0, 0, 3))[3 - i:23 - i] for i in range(4))).all()


def test_timers():
    """From the first kernel's begin to the last one's end"""
    c = Case([3000], 2, 4, 128, 4, "bf16", seed=10)
    g, timer = grads_of(c), kvb.Timer()
    for call in (lambda: run(c), lambda: backward(c, g)):
        call()
        timer.arm()
        call()
        assert 1.0 < timer.us() < 1e4
    timer.close()


def test_the_same_bits_and_a_replayed_graph():
    c = Case([70, 3, 130], 2, 4, 128, 4, "bf16", seed=5)
    g = grads_of(c)
    ta, sq = c.taps(), kvb.seqs(c.start, c.N, c.n_slots, slot=c.slot)
    want = backward(c, g)
    again = backward(c, g)
    assert all(torch.equal(want[n], again[n]) for n in want if want[n] is not None)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = backward(c, g, stream=side)
    assert all(torch.equal(want[n], again[n]) for n in want if want[n] is not None)
    r = {n: torch.empty_like(y) for n, y in want.items() if y is not None}
    work = torch.empty(kvb.conv_backward_work(c.sh, ta, sq), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kvb.kvb_conv_backward(c.sh, ta, sq, c.x, c.a, c.b, c.state0, g["dq"], g["dk"], g["dv"], g["dg"], g["dbeta"], g["dstate1"], r["dx"], r["da"], r["db"],
                              r["dweight"], None, r["dA_log"], r["ddt_bias"], r["dstate0"], work)
    for _ in range(3):
        for y in list(r.values()) + [work]:
            y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[n], r[n]) for n in r)


def test_differences():
    """The change of a weighted sum of all results along a random direction of all inputs, fp32: kvb_conv on both sides.

    Central differences at h = 2^-6 of a sum of some 1e4 terms, each result good to about 16 U: what rounding leaves is below
    16 U sqrt(sum of squared weighted results) / h, taken ten times; what h leaves, a third derivative, is taken out by a second difference at 2 h
    (Richardson) down to the fifth derivative's h^4 times the slope."""
    c = Case([9, 0, 40, 3], 2, 4, 32, 4, "f32", seed=6, bias=True)
    g = grads_of(c)
    r = backward(c, g)
    names = {"x": "dx", "a": "da", "b": "db", "weight": "dweight", "bias": "dbias", "A_log": "dA_log", "dt_bias": "ddt_bias", "state0": "dstate0"}
    gen = torch.Generator().manual_seed(2)
    way = {n: 0.1 * torch.randn(getattr(c, n).shape, generator=gen).cuda() for n in names}
    slope = sum(float((way[n].double() * r[m].double()).sum()) for n, m in names.items())
    base = {n: getattr(c, n).clone() for n in names}

    def total(h):
        for n in names:
            getattr(c, n).copy_(base[n] + h * way[n])
        o, s1 = run(c)
        return [(y.double(), g[m].double()) for y, m in zip(o + [s1], ("dq", "dk", "dv", "dg", "dbeta", "dstate1"))]

    h = 2.0 ** -6
    size = sum(float((y * w).square().sum()) for y, w in total(0.0)) ** 0.5

    def difference(h):
        return sum(float(((y - z) * w).sum()) for (y, w), (z, _) in zip(total(h), total(-h))) / (2 * h)

    got = (4 * difference(h) - difference(2 * h)) / 3
    # (moved inputs are rounded too: half a U of each, times its gradient)
    moved = sum(float((base[n].double() * r[m].double()).square().sum()) for n, m in names.items()) ** 0.5
    assert abs(got - slope) < 10 * (16 * U * size + U * moved) / h + 100 * h ** 4 * abs(slope)
