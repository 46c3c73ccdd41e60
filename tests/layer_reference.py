"""kvb_conv, kvb_norm and their gradients from the formulas, in 64 bits, token by token, with bounds of what fp32 may be off by."""
import torch

from running_error import V, cat, inverse_root, sigmoid, where


def f64(x):
    return None if x is None else V(x.detach().cpu().double())


def zeros(*size):
    return V(torch.zeros(*size, dtype=torch.float64))


def softplus(y):
    """max(y, 0) + log1p(exp(-|y|)): an exponential (2 units and the rounding of its argument), log1p (2), the sum"""
    v = torch.logaddexp(y.v, torch.zeros_like(y.v))
    return V(v, torch.sigmoid(y.v) * y.e + 6.0 * v)


def exact_sigmoid(y):
    s = torch.sigmoid(y.v)
    return V(s, s * (1.0 - s) * (y.e + 4.0) + 3.0 * s)


def gates(a, b, A_log, dt_bias):
    rate = f64(A_log).of(torch.exp, A_log.cpu().double().exp(), 2.0)
    y = f64(a) + f64(dt_bias)
    return V(-rate.v, rate.e), y, exact_sigmoid(f64(b))


class Conv:
    """One sequence (or one draft's root path): E are rows [W - 1 + n, C]"""

    def __init__(self, E, weight, bias, heads, n_unit, d, eps, unit=True):
        W = weight.shape[1]
        n = E.v.shape[0] - (W - 1)
        self.E, self.w, self.d, self.W, self.n = E, f64(weight), d, W, n
        z = zeros(n, E.v.shape[1]) if bias is None else V(f64(bias).v.expand(n, -1))
        for i in range(W):
            z = z + V(self.w.v[:, i]) * E[i:i + n]
        self.z = z
        self.s = sigmoid(z)
        self.y = z * self.s
        h = V(self.y.v.unflatten(-1, (heads, d)), self.y.e.unflatten(-1, (heads, d)))
        self.is_unit = (torch.arange(heads) < (n_unit if unit else 0))[None, :, None]
        sq = (h * h).sum(-1, d)
        self.r = where(self.is_unit, inverse_root(V(sq.v + eps, sq.e + sq.v + eps)), V(torch.ones_like(sq.v)))
        self.h = h
        self.n_out = where(self.is_unit, h * self.r, h)   # [n, heads, d]

    def backward(self, dn, dlast):
        """dz and dE from the gradients [n, heads, d] of the outputs and [W - 1, C] of E's last rows"""
        dot = (self.h * dn).sum(-1, self.d)
        c = self.r * self.r * self.r * dot
        dy = where(self.is_unit, self.r * dn - c * self.h, dn)
        dy = V(dy.v.flatten(1), dy.e.flatten(1))
        one = V(torch.ones_like(self.s.v))
        self.dz = dy * (self.s + self.y * (one - self.s))
        dE = zeros(*self.E.v.shape)
        for i in range(self.W):
            term = V(self.w.v[:, i]) * self.dz
            dE = dE + cat([zeros(i, term.v.shape[1]), term, zeros(self.W - 1 - i, term.v.shape[1])], 0)
        return dE if dlast is None else dE + cat([zeros(self.n, dlast.v.shape[1]), dlast], 0)


def norm(s, weight, gate, eps):
    """out, and what the gradients need"""
    sq = (s * s).sum(-1, s.v.shape[-1])
    w = s.v.shape[-1]
    r = inverse_root(V(sq.v / w + eps, sq.e / w + 2.0 * sq.v / w + eps))
    h = s * r
    out = h * f64(weight)
    act = None
    if gate is not None:
        t = sigmoid(f64(gate))
        act = f64(gate) * t
        out = out * act
    return out, r, h, act


def norm_backward(s, weight, gate, eps, dout, dsum, scale, rows_added):
    out, r, h, act = norm(s, weight, gate, eps)
    w, d = f64(weight), f64(dout)
    dc = d if act is None else d * act
    dh = dc * w
    width = s.v.shape[-1]
    dot = (dh * s).sum(-1, width)
    mean = dot * r
    mean = V(mean.v / width, mean.e / width + 2.0 * mean.v.abs() / width)
    ds = r * (dh - h * mean)
    if dsum is not None:
        ds = ds + f64(dsum)
    res = {"dres": ds, "dx": ds * V(torch.full_like(ds.v, scale)), "dweight": (dc * h).sum((0, 1), rows_added, keepdim=False)}
    if gate is not None:
        t, g = sigmoid(f64(gate)), f64(gate)
        one = V(torch.ones_like(t.v))
        res["dgate"] = d * (h * w) * (t * (g * (one - t) + one))
    return res
