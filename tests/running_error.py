"""Values in 64 bits with a bound of what fp32 arithmetic may be off by, carried along operation by operation (first order).

An operation of fp32 rounds by at most U = 2^-24 of its result; the hardware's exp2, reciprocal and inverse root by one unit in the last place, 2 U.
`e` counts in U.  A sum adds its terms one after the other at worst: as many roundings of the sum of magnitudes as it has additions.
"""
import torch

U = 2.0 ** -24


class V:
    def __init__(self, v, e=None):
        self.v = v
        self.e = torch.zeros_like(v) if e is None else e

    def __add__(self, o):
        v = self.v + o.v
        return V(v, self.e + o.e + v.abs())

    def __sub__(self, o):
        return self + V(-o.v, o.e)

    def __mul__(self, o):
        v = self.v * o.v
        return V(v, self.v.abs() * o.e + o.v.abs() * self.e + v.abs())

    def of(self, f, slope, units):
        """f(self), whose own rounding is `units` of the result"""
        v = f(self.v)
        return V(v, slope.abs() * self.e + units * v.abs())

    def sum(self, dim, additions, keepdim=True):
        return V(self.v.sum(dim, keepdim=keepdim), self.e.sum(dim, keepdim=keepdim) + additions * self.v.abs().sum(dim, keepdim=keepdim))

    def __getitem__(self, i):
        return V(self.v[i], self.e[i])


def where(c, a, b):
    return V(torch.where(c, a.v, b.v), torch.where(c, a.e, b.e))


def cat(vs, dim):
    return V(torch.cat([x.v for x in vs], dim), torch.cat([x.e for x in vs], dim))


def sigmoid(z):
    """rcp(1 + exp2(-log2(e) z)): the argument is off by two roundings of |z|, which moves the result by s (1 - s); exp2, the sum, rcp.
    The reciprocal of a number above 2^126 is below fp32's normal numbers and becomes 0: off by up to 2^-126, which what it is
    multiplied by (z, some hundreds at most there) makes larger."""
    s = torch.sigmoid(z.v)
    return V(s, s * (1.0 - s) * (z.e + 2.0 * z.v.abs() + 2.0) + 3.0 * s + 2.0 ** -126 / U)


def inverse_root(x):
    r = x.v ** -0.5
    return V(r, 0.5 * r / x.v * x.e + 2.0 * r)


def check(got, want, what):
    """got, of any type, against want: what fp32 may be off by, and the last rounding to got's type"""
    g = got.detach().cpu().double()
    f = torch.finfo(got.dtype)
    half = (f.eps / 2 if got.dtype != torch.float32 else 0.0) * want.v.abs() + f.smallest_normal * f.eps / 2
    allowed = U * want.e * (1.0 + 2.0 ** -7) + half + 1e-37   # (terms of second order; fp32's smallest numbers)
    off = (g - want.v).abs()
    bad = ~(off <= allowed)
    assert not bad.any(), "%s: %d of %d values, off by up to %.3g times what is allowed" % (
        what, int(bad.sum()), bad.numel(), float((off / allowed).nan_to_num(1e30)[bad].max()))
