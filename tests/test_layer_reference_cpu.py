"""The formulas in 64 bits that kvb_conv and kvb_norm are tested with, pinned to torch's own differentiation; and their bounds to fp32 arithmetic on the CPU."""
import torch

import layer_reference as ref
from running_error import U, V

HEADS, UNIT, D, W, EPS = 5, 3, 8, 4, 1e-6


def conv(E, w, bias, unit=True):
    n = E.shape[0] - (W - 1)
    z = sum(w[:, i] * E[i:i + n] for i in range(W)) + bias
    y = (z * torch.sigmoid(z)).unflatten(1, (HEADS, D))
    if not unit:
        return y
    return torch.cat([y[:, :UNIT] / (y[:, :UNIT].square().sum(-1, keepdim=True) + EPS).sqrt(), y[:, UNIT:]], 1)


def test_convolution():
    torch.manual_seed(0)
    for unit in (True, False):
        E, w, bias = (torch.randn(*s, dtype=torch.float64).float() for s in ((W - 1 + 20, HEADS * D), (HEADS * D, W), (HEADS * D,)))
        dn, dlast = torch.randn(20, HEADS, D), torch.randn(W - 1, HEADS * D)
        leaves = [x.double().requires_grad_(True) for x in (E, w, bias)]
        out = conv(*leaves, unit)
        dE, dw, dbias = torch.autograd.grad([out, leaves[0][-(W - 1):]], leaves, [dn.double(), dlast.double()])
        r = ref.Conv(ref.f64(E), w, bias, HEADS, UNIT, D, EPS, unit)
        got = r.backward(ref.f64(dn), ref.f64(dlast))
        assert torch.allclose(r.n_out.v, out.detach(), rtol=1e-12, atol=1e-12) and torch.allclose(got.v, dE, rtol=1e-12, atol=1e-12)
        assert torch.allclose(torch.stack([(r.dz.v * E.double()[i:i + 20]).sum(0) for i in range(W)], 1), dw, rtol=1e-12, atol=1e-12)
        assert torch.allclose(r.dz.v.sum(0), dbias, rtol=1e-12, atol=1e-12)
        # torch's fp32 stays within the bounds, and they are no more than some hundred times what it is off by
        x = [y.clone().requires_grad_(True) for y in (E, w, bias)]
        low = conv(*x, unit)
        dE32, = torch.autograd.grad([low, x[0][-(W - 1):]], x[:1], [dn, dlast])
        for a, b in ((low.detach(), r.n_out), (dE32, got)):
            off = (a.double() - b.v).abs()
            assert (off <= 1.02 * U * b.e).all() and U * b.e.mean() < 300 * off.mean()


def test_norm():
    torch.manual_seed(1)
    x, gate, dout, dsum = (torch.randn(7, 3, 40) for _ in range(4))
    w = torch.randn(40)
    for g in (None, gate):
        leaves = [y.double().requires_grad_(True) for y in (x, w) + ((g,) if g is not None else ())]
        out = leaves[0] / (leaves[0].square().mean(-1, keepdim=True) + EPS).sqrt() * leaves[1]
        if g is not None:
            out = out * leaves[2] * torch.sigmoid(leaves[2])
        grads = torch.autograd.grad(out, leaves, dout.double())
        got = ref.norm_backward(ref.f64(x), w, g, EPS, dout, dsum, 0.5, 21)
        assert torch.allclose(ref.norm(ref.f64(x), w, g, EPS)[0].v, out.detach(), rtol=1e-12, atol=1e-12)
        want = {"dres": grads[0] + dsum.double(), "dx": 0.5 * (grads[0] + dsum.double()), "dweight": grads[1]}
        if g is not None:
            want["dgate"] = grads[2]
        assert set(want) == set(got)
        assert all(torch.allclose(got[n].v, want[n], rtol=1e-12, atol=1e-12) for n in want)


def test_gates():
    torch.manual_seed(2)
    a, b, A_log, dt_bias = 5 * torch.randn(50, 3), 5 * torch.randn(50, 3), torch.randn(3), torch.randn(3)
    rate, y, beta = ref.gates(a, b, A_log, dt_bias)
    want = -A_log.double().exp() * torch.nn.functional.softplus(a.double() + dt_bias.double(), threshold=1e9)
    assert torch.allclose((rate * ref.softplus(y)).v, want, rtol=1e-12) and torch.allclose(beta.v, torch.sigmoid(b.double()), rtol=1e-12)


def test_bounds_of_operations():
    """A sum of products, operation by operation in fp32"""
    torch.manual_seed(3)
    a, b = torch.randn(1000, 16), torch.randn(1000, 16)
    s = torch.zeros(1000)
    for i in range(16):
        s = s + a[:, i] * b[:, i]
    want = (V(a.double()) * V(b.double())).sum(1, 16, keepdim=False)
    assert ((s.double() - want.v).abs() <= U * want.e).all()
