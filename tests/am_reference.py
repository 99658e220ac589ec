"""The acoustic-model operators from their definitions, in float64 on the CPU,
and the error bounds their tests use.

Bounds.  u(T) is the unit roundoff of an output type: one rounding to nearest
moves a value v by at most u |v| (or half the spacing of the subnormals).  A
float32 sum of n terms t_i moves by at most LAMBDA sqrt(n) 2^-24 sum |t_i| but
for a vanishing probability (roundings as independent errors of mean zero;
Higham and Mary 2019, with lambda = 8), plus two more roundings of the terms'
size for the products and scales around it.  Operands that are themselves
rounded to u relative each move a sum by at most LAMBDA u sqrt(sum t_i^2) in
the same sense.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
U32 = 2.0 ** -24
LAMBDA = 8.0
E4M3_MAX = 448.0


def sum_bound(n, magnitude):
    """Error of a float32 sum of n terms whose magnitudes sum to `magnitude`."""
    return (LAMBDA * math.sqrt(max(n, 1)) + 4) * U32 * magnitude


def d(t):
    return None if t is None else t.detach().cpu().double()


def act(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    if kind == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2.0)))
    return z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    if kind == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s + z * s * (1 - s)
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2.0))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


# |act'| and |slope'| are at most these
ACT_LIPSCHITZ = 1.13


def linear(x, w, bias, kind, residual, x_scale=None, w_scale=None):
    """(y, z, bound on z's error before its rounding)."""
    x, w = d(x), d(w)
    z, mag = x @ w.t(), x.abs() @ w.abs().t()
    if x_scale is not None:
        s = d(x_scale)[:, None] * d(w_scale)
        z, mag = z * s, mag * s
    if bias is not None:
        z, mag = z + d(bias), mag + d(bias).abs()
    y = act(z, kind)
    if residual is not None:
        y = y + d(residual)
    return y, z, sum_bound(x.shape[1], mag)


def norm(x, residual, gain, eps):
    s = d(x) + (d(residual) if residual is not None else 0)
    r = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    return s, s * r * (d(gain) if gain is not None else 1)


def norm_backward(dy, s, gain, dsum, eps):
    dy, s = d(dy), d(s)
    r = 1 / torch.sqrt((s * s).mean(1, keepdim=True) + eps)
    u = dy * (d(gain) if gain is not None else 1)
    dx = r * u - r ** 3 * s * (u * s).mean(1, keepdim=True)
    if dsum is not None:
        dx = dx + d(dsum)
    return dx, (dy * s * r).sum(0)


def distill(logits, index, top, temperature, weight):
    """Row by row: (loss, lse, dlogits)."""
    x, top = d(logits), d(top)
    rows, n = x.shape
    loss, lse, dl = torch.zeros(rows).double(), torch.zeros(rows).double(), torch.zeros(rows, n).double()
    for m in range(rows):
        w = 1.0 if weight is None else float(weight[m])
        lse[m] = torch.logsumexp(x[m] / temperature, 0)
        used = [j for j in range(index.shape[1]) if 0 <= int(index[m, j]) < n and top[m, j] > -math.inf]
        if w == 0 or not used:
            continue
        p = torch.softmax(top[m, used] / temperature, 0)
        log_q = x[m] / temperature - lse[m]
        g = torch.exp(log_q)
        total = 0.0
        for pj, j in zip(p, used):
            i = int(index[m, j])
            if pj > 0:
                total += float(pj) * (math.log(float(pj)) - float(log_q[i]))
            g[i] -= pj
        loss[m], dl[m] = w * temperature ** 2 * total, w * temperature * g
    return loss, lse, dl


def loglikes(logits, log_prior, scale):
    x = d(logits)
    p = d(log_prior) if log_prior is not None else torch.zeros(x.shape[1]).double()
    ll = scale * (x - torch.logsumexp(x, 1, keepdim=True) - p)
    return torch.where((x == -math.inf) | (p == -math.inf), torch.full_like(x, -math.inf), ll)


def close(got, want, bound, tag):
    """Element by element; infinities and NaN in the same places."""
    got, bound = d(got), torch.as_tensor(bound).double().expand(want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN in other places" % tag
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), "%s: infinities differ" % tag
    off = (got - want).abs()
    bad = fine & ~(off <= bound)
    if bad.any():
        at = torch.nonzero(bad)[0].tolist()
        raise AssertionError("%s: %d of %d values off; at %s got %r, want %r, allowed %r" % (
            tag, int(bad.sum()), bad.numel(), at, float(got[tuple(at)]), float(want[tuple(at)]),
            float(bound[tuple(at)])))
