"""The layer norm, the gated layer and the clipping of gradients from their
definitions, in float64 on the CPU, and the error bounds their tests use (u, LAMBDA
and sum_bound: am_reference.py)."""
import math

import torch

import am_reference as R
from am_reference import U32, d


def ones(t, like):
    return torch.ones(like, dtype=torch.float64) if t is None else d(t)


class Moments:
    """Mean, differences and reciprocal deviation of rows s, and the bounds of their
    errors in float32: `off` is the error of s itself.

    The mean is m0 + c, c the mean of the differences from m0: it is off by what
    summing the differences leaves, sum_bound(D, sum|s - mean|) / D, and by the mean
    of s's own errors.  A difference is two subtractions' roundings more.  The
    variance is off by summing's relative (LAMBDA sqrt(D) + 4) u, the differences'
    roundings (twice 2 u) and s's errors, relatively 2 rms(off) r; its root by half
    of that, and by a root, a sum, a division and a quotient: 6 u more."""

    def __init__(self, s, eps, off=None):
        s = d(s)
        n = s.shape[1]
        off = torch.zeros_like(s) if off is None else off
        mean = s.mean(1, keepdim=True)
        self.diff = s - mean
        var = (self.diff ** 2).mean(1, keepdim=True)
        self.r = 1 / torch.sqrt(var + eps)
        self.h = self.diff * self.r
        size = self.diff.abs().mean(1, keepdim=True)
        e_mean = R.sum_bound(n, size * n) / n + off.mean(1, keepdim=True)
        e_diff = off + e_mean + 3 * U32 * self.diff.abs()
        self.rel = ((R.LAMBDA * math.sqrt(n) + 8) * U32 + 2 * off.pow(2).mean(1, keepdim=True).sqrt() * self.r) / 2 + 6 * U32
        self.err = self.r * e_diff + self.h.abs() * self.rel   # of h


def layer_norm(x, residual, gain, bias, eps):
    """(s, v, bound on v's error before its rounding)."""
    s = d(x) + (d(residual) if residual is not None else 0)
    mo = Moments(s, eps, U32 * s.abs() if residual is not None else None)
    g = ones(gain, s.shape[1])
    v0 = mo.h * g
    v = v0 + (d(bias) if bias is not None else 0)
    return s, v, mo.err * g.abs() + U32 * (v0.abs() + v.abs()) * 1.01


def layer_norm_backward(dy, s, gain, dsum, eps):
    """(dx, dgain, dbias, bounds on the errors of each before a rounding).

    mean(u) and mean(u h) are sums of n terms, each with a product's roundings;
    h's error reaches the second through every term and dx once more through h."""
    dy, n, m = d(dy), s.shape[1], s.shape[0]
    mo = Moments(s, eps)
    u = dy * ones(gain, n)
    mean_u, mean_uh = u.mean(1, keepdim=True), (u * mo.h).mean(1, keepdim=True)
    inner = u - mean_u - mo.h * mean_uh
    dx = mo.r * inner
    e_mean = (R.sum_bound(n, u.abs().sum(1, keepdim=True)) / n + 2 * U32 * mean_u.abs())
    e_mean_uh = (R.sum_bound(n, (u * mo.h).abs().sum(1, keepdim=True)) / n + (u.abs() * mo.err).mean(1, keepdim=True)
                 + 6 * U32 * (u * mo.h).abs().mean(1, keepdim=True))
    err = mo.r * (2 * U32 * u.abs() + e_mean + mo.h.abs() * e_mean_uh + mo.err * mean_uh.abs()
                  + 4 * U32 * (u.abs() + mean_u.abs() + (mo.h * mean_uh).abs())) + mo.rel * dx.abs()
    if dsum is not None:
        dx = dx + d(dsum)
        err = err + U32 * dx.abs()
    dg, db = (dy * mo.h).sum(0), dy.sum(0)
    e_dg = R.sum_bound(m, (dy * mo.h).abs().sum(0)) + (dy.abs() * mo.err).sum(0) * 1.01
    return dx, dg, db, err, e_dg, R.sum_bound(m, dy.abs().sum(0))


def gated(x, w, bias, kind, x_scale=None, w_scale=None):
    """(y, z, bound on z's error, bound on y's, both before a rounding).  The activation is good to 8 u of its
    value and its argument, and its slope is at most ACT_LIPSCHITZ."""
    _, z, err = R.linear(x, w, bias, "none", None, x_scale, w_scale)
    n = z.shape[1] // 2
    a, v = R.act(z[:, :n], kind), z[:, n:]
    e_a = R.ACT_LIPSCHITZ * err[:, :n] + 8 * U32 * (a.abs() + z[:, :n].abs())
    y = a * v
    return y, z, err, e_a * v.abs() + a.abs() * err[:, n:] + e_a * err[:, n:] + U32 * y.abs()


def gated_dz(dy, pre, kind):
    """(dz, bound on its error): products' roundings, and a slope and an activation good to 16 u (1 + |gate|)."""
    dy, pre = d(dy), d(pre)
    n = dy.shape[1]
    gate, value = pre[:, :n], pre[:, n:]
    dz = torch.cat([dy * value * R.slope(gate, kind), dy * R.act(gate, kind)], 1)
    loose = 16 * U32 * (1 + gate.abs()) * dy.abs()
    return dz, torch.cat([loose * value.abs(), loose], 1)


# what two 16-bit values leave of dz: relative, absolute
LEFT = {torch.bfloat16: (2.0 ** -16, 0.0), torch.float16: (2.0 ** -22, 2.0 ** -35)}


def product(a, b, slack, rel, least, tiny):
    """(a b, bound) where a is held to `slack`, and to rel of it or least besides, as independent errors."""
    want = a @ b
    err = R.sum_bound(2 * a.shape[1], a.abs() @ b.abs()) + (slack + least) @ b.abs()
    return want, err + R.LAMBDA * rel * torch.sqrt((a * a) @ (b * b)) + tiny * b.abs().sum(0)
