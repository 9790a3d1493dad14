"""The channel products and 8-bit checkpoints from their definitions, in 64 bits on the CPU, and how far a 32-bit
computation may be from them."""
from __future__ import annotations

import math

import numpy as np
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8            # half a unit in the last place of 24 and 8 bits, relative
BLOCK = 32


def unit(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def act(z, name):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), z)
    if name == "gelu":
        return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return torch.where(z <= 0, torch.zeros_like(z), torch.ones_like(z))
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    return torch.ones_like(z)


def forward(x, w, b, r, name, dtype):
    """(z, y, bound on z's error, bound on y's) of f64 inputs that hold values of `dtype`.

    A sum of K products in 32 bits, in any order, is off by at most about (K + 8) half units of the sum of the
    magnitudes.  The activations' slopes are at most 1.13 in size; they are computed to 8 half units of 1 + |z| (f32) or,
    for results that are rounded to bf16, to 1e-6 (1 + |z|); each output is rounded once."""
    z = x @ w.T
    size = x.abs() @ w.abs().T
    if b is not None:
        z, size = z + b, size + b.abs()
    z_off = (x.shape[1] + 8) * U32 * size + 1e-38
    y = act(z, name)
    y_off = z_off * (1.13 if name != "none" else 1.0)
    if name in ("gelu", "silu"):
        y_off = y_off + (1e-6 if dtype == torch.bfloat16 else 8 * U32) * (1 + z.abs())
    if r is not None:
        y = y + r
        y_off = y_off + U32 * y.abs()
    return z, y, z_off, y_off * (1 + unit(dtype)) + unit(dtype) * y.abs()


def backward(g, x, z, w, name, dtype):
    """((dx, dw, db), their bounds) from x and z as they are held: dz = g act'(z) to 1e-6 |g| (1 + |z|) (bf16) or 8 half
    units of it (f32), rounded to the dtype before the products (not before the sum that is db)."""
    s = slope(z, name)
    dz = g * s
    dz_off = torch.zeros_like(dz)
    if name in ("gelu", "silu"):
        dz_off = (1e-6 if dtype == torch.bfloat16 else 16 * U32) * g.abs() * (1 + z.abs())
    kept = dz_off + (unit(dtype) * dz.abs() if name != "none" else 0)
    big = dz.abs() + dz_off
    u = unit(dtype)

    def bound(v, off, size, terms):
        off = off + (terms + 8) * U32 * size + 1e-38
        return off * (1 + u) + u * v.abs()
    dx, dw, db = dz @ w, dz.T @ x, dz.sum(0)
    return (dx, dw, db), (bound(dx, kept @ w.abs(), big @ w.abs(), w.shape[0]),
                          bound(dw, kept.T @ x.abs(), big.T @ x.abs(), g.shape[0]),
                          bound(db, dz_off.sum(0), big.sum(0), g.shape[0]))


def checkpoint8(v):
    """(codes, bytes) of an f64 or f32 numpy array [rows, n] by the definition."""
    v = np.asarray(v, np.float64)
    rows, n = v.shape
    codes, exps = np.zeros((rows, n), np.int8), np.zeros((rows, -(-n // BLOCK)), np.uint8)
    for j in range(exps.shape[1]):
        part = v[:, j * BLOCK:(j + 1) * BLOCK]
        fine = np.isfinite(part)
        top = np.maximum(np.where(fine, np.abs(part), 0.0).max(1), 2.0 ** -120)
        e = np.frexp(top)[1] - 7                           # frexp's fraction is in [1/2, 1)
        q = np.clip(np.rint(np.ldexp(np.where(fine, part, 0.0), -e[:, None])), -127, 127)
        codes[:, j * BLOCK:(j + 1) * BLOCK] = np.where(fine, q, -128)
        exps[:, j] = e + 127
    return codes, exps


def restored(codes, exps):
    e = np.repeat(exps.astype(np.int64) - 127, BLOCK, 1)[:, :codes.shape[1]]
    return np.where(codes == -128, np.nan, np.ldexp(codes.astype(np.float64), e))


def bits(z):
    """int32 sign words of f64 z [rows, n]: a bit set where not z <= 0."""
    rows, n = z.shape
    w = np.zeros((rows, -(-n // BLOCK) * BLOCK), np.uint64)
    w[:, :n] = ~(np.asarray(z) <= 0)
    w = (w.reshape(rows, -1, BLOCK) << np.arange(BLOCK, dtype=np.uint64)).sum(-1)
    return w.astype(np.uint32).view(np.int32)


def within(got, want, off, what):
    got = got.detach().double().cpu()
    bad = ~((got - want).abs() <= off)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    if bad.any():
        i = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d values off, first at %r: %.9g for %.9g, at most %.3g allowed"
                             % (what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(off[i])))
