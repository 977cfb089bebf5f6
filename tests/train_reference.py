"""Plain 64-bit forms of the operators around an MLP block's products, with bounds of the error of an fp32 evaluation beside them.

A bound counts roundings of 2^-24 (E), one for every operation on the way; SUM of them for a sum over a row, which a lane's 16 terms, the six
steps over a wave, four over waves and the last division make; a sum over R rows in any order R.  Errors of inputs of a step are passed on by its
derivative."""
from __future__ import annotations

import math

import torch

E = 2.0 ** -24
SUM = 32
LAYER, RMS = 0, 1


class Norm:
    def __init__(self, kind, eps, gamma=None, beta=None):
        self.kind, self.eps, self.gamma, self.beta = kind, eps, gamma, beta

    def weights(self, n):
        one = torch.ones(n, dtype=torch.float64)
        return one if self.gamma is None else self.gamma, 0 * one if self.beta is None else self.beta


def statistics(v, norm):
    mean = v.mean(-1, keepdim=True) if norm.kind == LAYER else torch.zeros_like(v[:, :1])
    return mean, 1.0 / torch.sqrt(((v - mean) ** 2).mean(-1, keepdim=True) + norm.eps)


def normalise(v, dv, norm):
    """norm(v), mean, rstd and the bounds of their errors, dv the bound of v's."""
    mean, rstd = statistics(v, norm)
    gamma, beta = norm.weights(v.shape[1])
    size = v.abs().mean(-1, keepdim=True)
    d = v - mean
    var = (d ** 2).mean(-1, keepdim=True)
    off = dv.mean(-1, keepdim=True) + (SUM + 8) * E * size if norm.kind == LAYER else torch.zeros_like(mean)
    # the squares: their inputs' errors, their own sums; the waves' means are off by fractions of the row's size
    dvar = 2 * (d.abs() * (dv + off)).mean(-1, keepdim=True) + (SUM + 16) * E * var + 2 * var.sqrt() * off + 2 * off ** 2 + (dv ** 2).mean(-1, keepdim=True)
    low = torch.clamp(var + norm.eps - dvar, min=0.0)
    rel = dvar / (2 * torch.clamp(low, min=1e-300)) + 4 * E
    hat = d * rstd
    dhat = hat.abs() * (rel + 3 * E) + rstd * (1 + rel) * (dv + off)
    y = hat * gamma + beta
    return y, mean, rstd, gamma.abs() * dhat + 2 * E * ((hat * gamma).abs() + y.abs()), off, rel * rstd


def residual_norm(x, r, post, gate, alpha, pre):
    """h, y, the statistics and bounds: a dict of (value, bound)."""
    out = {}
    t, dt = x, torch.zeros_like(x)
    if post:
        t, out_mean, out_rstd, dt, dm, dr = normalise(x, dt, post)
        out["mean1"], out["rstd1"] = (out_mean, dm), (out_rstd, dr)
    g = torch.ones(x.shape[1], dtype=torch.float64) if gate is None else gate
    h = alpha * r + g * t
    dh = g.abs() * dt + 2 * E * (alpha * r).abs() + E * h.abs()
    out["h"] = (h, dh)
    if pre:
        y, mean, rstd, dy, dm, dr = normalise(h, dh, pre)
        out["y"], out["mean2"], out["rstd2"] = (y, dy), (mean, dm), (rstd, dr)
    return out


def standard_grad(g, dg, hat, rstd, kind):
    """rstd (g - mean g - hat mean(g hat)) of hat to 2 E."""
    s1 = g.mean(-1, keepdim=True) if kind == LAYER else torch.zeros_like(rstd)
    s2 = (g * hat).mean(-1, keepdim=True)
    ds1 = dg.mean(-1, keepdim=True) + (SUM + 2) * E * g.abs().mean(-1, keepdim=True) if kind == LAYER else s1
    ds2 = (dg * hat.abs()).mean(-1, keepdim=True) + (SUM + 6) * E * (g * hat).abs().mean(-1, keepdim=True)
    out = rstd * (g - s1 - hat * s2)
    return out, rstd * (dg + ds1 + hat.abs() * ds2 + 6 * E * (g.abs() + s1.abs() + (hat * s2).abs()))


def residual_norm_grad(x, post, gate, alpha, h, pre, dh, dy, stats):
    """stats: (mean1, rstd1, mean2, rstd2) as they were stored, columns.  A dict of (value, bound); the weights' gradients are over all rows given."""
    n, rows = x.shape[1], x.shape[0]
    out = {}
    one = torch.ones(n, dtype=torch.float64)
    d = torch.zeros_like(x) if dh is None else dh
    dd = torch.zeros_like(x)
    if pre:
        gamma, _ = pre.weights(n)
        hat = (h - (stats[2] if pre.kind == LAYER else 0.0)) * stats[3]
        g = dy * gamma
        s, ds = standard_grad(g, E * g.abs(), hat, stats[3], pre.kind)
        dd = ds + 2 * E * (d.abs() + (d + s).abs())
        d = d + s
        out["dgamma2"] = ((dy * hat).sum(0), (rows + 20) * E * (dy * hat).abs().sum(0))
        out["dbeta2"] = (dy.sum(0), (rows + 16) * E * dy.abs().sum(0))
    out["dr"] = (alpha * d, abs(alpha) * dd + 2 * E * (alpha * d).abs())
    g = one if gate is None else gate
    gamma, beta = post.weights(n) if post else (one, 0 * one)
    hat = (x - (stats[0] if post.kind == LAYER else 0.0)) * stats[1] if post else x
    a, b = (d * hat).sum(0), d.sum(0)
    da = (dd * hat.abs()).sum(0) + (rows + 20) * E * (d * hat).abs().sum(0)
    db = dd.sum(0) + (rows + 16) * E * d.abs().sum(0)
    out["dgate"] = (gamma * a + beta * b, gamma.abs() * da + beta.abs() * db + 4 * E * ((gamma * a).abs() + (beta * b).abs()))
    e = d * g * gamma
    de = (g * gamma).abs() * dd + 3 * E * e.abs()
    if post:
        out["dgamma1"] = (g * a, g.abs() * da + 2 * E * (g * a).abs())
        out["dbeta1"] = (g * b, g.abs() * db + 2 * E * (g * b).abs())
        out["dx"] = standard_grad(e, de, hat, stats[1], post.kind)
    else:
        out["dx"] = (e, de)
    return out


def gelu(a):
    return 0.5 * a * torch.erfc(-a * math.sqrt(0.5))


def gelu_slope(a):
    return 0.5 * torch.erfc(-a * math.sqrt(0.5)) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
