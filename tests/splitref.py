"""Products of f32 values with one term a sum, so that each has one right value whatever the order, and which a computation
from bf16 parts gets right only if it takes every one of the partial products that it says it takes."""
from __future__ import annotations

import torch


def _mantissas(shape, bits, gen):
    """Odd multiples of 2^(1 - bits) in [1, 2), with signs."""
    v = torch.randint(1 << (bits - 2), 1 << (bits - 1), shape, generator=gen, dtype=torch.int64) * 2 + 1
    sign = torch.randint(0, 2, shape, generator=gen, dtype=torch.int64) * 2 - 1
    return (v * sign).double() * 2.0 ** (1 - bits)


def one_term(rows_a, rows_b, contraction, seed, ones=False):
    """(A [rows_a, contraction], B [rows_b, contraction], A B^T), all f32 and exact: a row of B has one value that is not
    zero, somewhere.  By contraction index in turn, A has 24 bits and B one, or A one and B 24, or both 12; ones: A has
    24 bits and B +-1 throughout."""
    gen = torch.Generator().manual_seed(seed)
    at = torch.randint(0, contraction, (rows_b,), generator=gen)
    at[:min(rows_b, 3)] = torch.tensor([0, contraction - 1, contraction // 2])[:rows_b]
    kind = torch.zeros(contraction, dtype=torch.int64) if ones else torch.arange(contraction) % 3
    bits_a, bits_b = torch.tensor([24, 2, 12]), torch.tensor([2, 24, 12])

    def values(rows, bits, kinds):
        out = torch.empty(rows, len(kinds), dtype=torch.float64)
        for i in range(3):
            mine = kinds == i
            v = _mantissas((rows, int(mine.sum())), int(bits[i]), gen)
            out[:, mine] = v.sign() if bits[i] == 2 else v
        return out
    a = values(rows_a, bits_a, kind)
    hot = values(1, bits_b, kind[at])[0]
    b = torch.zeros(rows_b, contraction, dtype=torch.float64)
    b[torch.arange(rows_b), at] = hot
    d = a[:, at] * hot
    assert torch.equal(d.float().double(), d) and torch.equal(a.float().double(), a) and torch.equal(b.float().double(), b)
    return a.float(), b.float(), d.float()


def parts(v):
    """h, m, l: three bf16 values that add up to f32 v."""
    out = []
    for _ in range(3):
        p = v.bfloat16().float()
        out.append(p)
        v = v - p
    return out


def from_parts(a, b, left_out=()):
    """A B^T from bf16 parts, the smallest orders first, without the products (i, j) in left_out."""
    pa, pb = parts(a), parts(b)
    d = torch.zeros(a.shape[0], b.shape[0])
    for order in (2, 1, 0):
        for i in range(order + 1):
            if (i, order - i) not in left_out:
                d = d + pa[i] @ pb[order - i].t()
    return d


def relative_error(got, want):
    """2-norm of the error over that of the 64-bit value."""
    return float((got.double() - want).norm() / want.norm())
