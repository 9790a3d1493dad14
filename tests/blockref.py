"""Residual borders and dropout from their definitions, in 64 bits on the CPU, each value with a bound on how far a 32-bit
computation may be from it."""
from __future__ import annotations

import math

import numpy as np
import torch

U32 = 2.0 ** -24
# Sums over a row: at most 16 values one after another in a lane, six steps over a wave, 16 waves; with what a product or
# a change of sign before them costs.
DEPTH = 48


def unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U32


class Off:
    """A value and how far the computed one may be from it: every operation in 32 bits is off by half a unit of its result
    (a few for the functions), and carries along what its operands are off by."""

    def __init__(self, v, e=0.0):
        self.v = v
        self.e = e if isinstance(e, torch.Tensor) else torch.full_like(v, e)

    def __add__(self, o):
        v = self.v + o.v
        return Off(v, self.e + o.e + U32 * v.abs())

    def __sub__(self, o):
        return self + Off(-o.v, o.e)

    def __mul__(self, o):
        v = self.v * o.v
        return Off(v, self.v.abs() * o.e + self.e * o.v.abs() + self.e * o.e + U32 * v.abs() + 2.0 ** -149)

    def sum(self, axis, depth):
        return Off(self.v.sum(axis, keepdim=True), self.e.sum(axis, keepdim=True) + depth * U32 * self.v.abs().sum(axis, keepdim=True))

    def mean(self):
        n = self.v.shape[-1]
        s = self.sum(-1, DEPTH)
        return Off(s.v / n, (s.e + 2 * U32 * s.v.abs()) / n)

    def rsqrt(self):
        v = self.v.rsqrt()
        # (first order, half as much again for what is beyond it while e is below a third of the value; 4 units for root and quotient)
        return Off(v, 0.75 * v * self.e / self.v + 4 * U32 * v)

    def rounded(self, dtype):
        """The bound of the value that is returned in dtype."""
        return self.v, self.e * (1 + unit(dtype)) + unit(dtype) * self.v.abs()


def logistic(z, dtype):
    """Of results that are rounded to bf16, exp2 and a reciprocal of the hardware: 1e-6 relative; 32 bits: 8 units.  (The
    argument's own rounding grows with it: half a unit of |z| is that much of the exponential.)"""
    v = torch.sigmoid(z.v)
    rel = (1e-6 if dtype == torch.bfloat16 else 8 * U32) + 4 * U32 * z.v.abs()
    return Off(v, v * (rel + z.e))


def normed(v, kind, w, b, eps):
    """(norm, normalised values, (mu, r))"""
    mu = v.mean() if kind == "layer" else Off(torch.zeros_like(v.v[..., :1]))
    c = v - mu if kind == "layer" else v
    r = ((c * c).mean() + Off(torch.full_like(mu.v, eps), U32 * eps)).rsqrt()
    h = c * r
    p = h if w is None else h * w
    return (p if b is None else p + b), h, (mu, r)


def normed_backward(g, h, r, kind, w):
    t = g if w is None else g * w
    d = t - h * (t * h).mean()
    if kind == "layer":
        d = d - t.mean()
    return d * r


def philox(seed, counter):
    """Ten rounds on an array [4, ...] of python-sized whole numbers, by the paper's definition."""
    c = [np.asarray(x, object) for x in counter]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rows, n, p, seed, offset):
    """Truth values [rows, n] and the factor of what is kept; rows: a count, or the rows' numbers."""
    rows = np.arange(rows) if isinstance(rows, int) else np.asarray(rows)
    q = math.floor(65536 * p + 0.5)
    groups = -(-n // 8)
    row, group = np.meshgrid(rows, np.arange(groups), indexing="ij")
    words = philox(seed & (1 << 64) - 1, [group, row, np.full_like(row, 0) + (offset & 0xFFFFFFFF), np.full_like(row, 0) + (offset >> 32)])
    u = np.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], -1).reshape(len(rows), groups * 8)[:, :n]
    return torch.from_numpy((u >= q).astype(bool)), (65536.0 / (65536 - q) if q < 65536 else 0.0)


def border(dtype, x, f=None, norm="none", weight=None, bias=None, gate=None, gate_act="none", scale=None, p=0.0, seed=0,
           offset=0, next_norm="none", next_weight=None, next_bias=None, eps=1e-6, dy=None, dh=None):
    """{name: (value, bound)} of the outputs and, with dy or dh, the gradients.  Tensors are rows [m, n] in f64; gate [g, n]
    with m a multiple of g.  f None: the next norm of x alone."""
    o = {}
    wrap = lambda t: None if t is None else Off(t)          # noqa: E731
    x, f, w, b, s, nw, nb = map(wrap, (x, f, weight, bias, scale, next_weight, next_bias))
    m, n = x.v.shape
    y = x
    if f is not None:
        P, fh, fs = (f, f, None) if norm == "none" else normed(f, norm, w, b, eps)
        G = slope = None
        if gate is not None:
            z = Off(gate.repeat_interleave(m // gate.shape[0], 0))
            G, slope = z, Off(torch.ones_like(z.v))
            if gate_act != "none":
                sg = logistic(z, dtype)
                one = Off(torch.ones_like(z.v))
                G, slope = (sg, sg * (one - sg)) if gate_act == "sigmoid" else (z * sg, sg * (one + z * (one - sg)))
        c = P if G is None else P * G
        c = c if s is None else c * s
        keep = None
        if p > 0:
            keep, factor = kept(m, n, p, seed, offset)
            drop = lambda t: Off(torch.where(keep, t.v * factor, 0.0), torch.where(keep, (t.e + 3 * U32 * t.v.abs()) * factor, 0.0))  # noqa: E731
            c = drop(c)
        y = x + c
        o["y"] = y.rounded(dtype)
    if next_norm != "none":
        h, yh, ys = normed(y, next_norm, nw, nb, eps)
        o["h"] = h.rounded(dtype)
    if dy is None and dh is None:
        return o
    rows = m + 48                    # sums over rows, in whatever order
    d = Off(torch.zeros_like(x.v)) if dy is None else Off(dy)
    if next_norm != "none":
        # the backward pass has y as it was rounded
        if f is not None:
            yh = Off(yh.v, yh.e + ys[1].v * unit(dtype) * y.v.abs())
        g = Off(torch.zeros_like(x.v)) if dh is None else Off(dh)
        d = d + normed_backward(g, yh, ys[1], next_norm, nw) if dh is not None else d
        o["dnext_weight"] = (g * yh).sum(0, rows).rounded(dtype)
        o["dnext_bias"] = g.sum(0, rows).rounded(dtype)
    o["dx"] = d.rounded(dtype)
    if f is None:
        return o
    t = drop(d) if keep is not None else d
    gp = t * P
    o["dscale"] = (gp if G is None else gp * G).sum(0, rows).rounded(dtype)
    ts = t if s is None else t * s
    if G is not None:
        dg = ts * P * slope
        o["dgate"] = Off(dg.v.view(gate.shape[0], -1, n), dg.e.view(gate.shape[0], -1, n)).sum(1, rows).rounded(dtype)
        o["dgate"] = tuple(v.squeeze(1) for v in o["dgate"])
    dP = ts if G is None else ts * G
    if norm == "none":
        o["df"] = dP.rounded(dtype)
    else:
        o["dweight"] = (dP * fh).sum(0, rows).rounded(dtype)
        o["dbias"] = dP.sum(0, rows).rounded(dtype)
        o["df"] = normed_backward(dP, fh, fs[1], norm, w).rounded(dtype)
    return o


def within(got, want, what):
    """A tensor within a (value, bound), flat vectors against [1, n]."""
    v, off = want
    got = got.detach().double().cpu().reshape(v.shape)
    bad = ~((got - v).abs() <= off + 1e-37)
    if bad.any():
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d values off, first at %r: %.9g for %.9g, at most %.3g allowed"
                             % (what, int(bad.sum()), bad.numel(), i, float(got[i]), float(v[i]), float(off[i])))
