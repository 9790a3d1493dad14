"""Values in 4 bits by their definition, on the CPU."""
from __future__ import annotations

import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
# borders between neighbouring values, and whether a value on the border goes up (to the even code)
BORDERS = ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False))


def save(v):
    """(codes [rows, 64 G], scale bytes [G, rows up to 4, 4]) of a [rows, n] array."""
    v = np.asarray(v, np.float64)
    rows, n = v.shape
    groups = -(-n // 128)
    pad = np.zeros((rows, groups * 128))
    pad[:, :n] = v
    blocks = pad.reshape(rows, groups * 4, 32)
    fine = np.isfinite(blocks).all(-1)
    top = np.maximum(np.where(fine, np.abs(np.where(fine[..., None], blocks, 0)).max(-1), 1), 2.0 ** -120)
    e = np.frexp(top)[1] - 3                              # frexp's fraction is in [1/2, 1)
    q = np.where(fine[..., None], np.ldexp(blocks, -e[..., None]), 0.0)
    code = sum(((np.abs(q) >= b) if up else (np.abs(q) > b)).astype(int) for b, up in BORDERS)
    code = code + 8 * (np.signbit(blocks) & fine[..., None])
    code = code.reshape(rows, groups * 128)
    byte = np.where(fine, e + 127, 255)
    byte[:, -(-n // 32):] = 127
    exps = np.full((groups, -(-rows // 4) * 4, 4), 127, np.uint8)
    exps[:, :rows] = byte.reshape(rows, groups, 4).transpose(1, 0, 2)
    return (code[:, ::2] | code[:, 1::2] << 4).astype(np.uint8), exps


def load(codes, exps, n):
    rows = codes.shape[0]
    c = np.stack((codes & 15, codes >> 4), -1).reshape(rows, -1).astype(int)
    v = np.where(c >= 8, -1.0, 1.0) * VALUES[c & 7]
    byte = exps[:, :rows].transpose(1, 0, 2).reshape(rows, -1).astype(int).repeat(32, 1)
    return np.where(byte == 255, np.nan, np.ldexp(v, byte - 127))[:, :n]
