"""Values in 4 bits and products of them, for serving what ``linear`` has trained.

``tv_quantize4`` holds a tensor in blocks of 32 values with a common power of two, a bit over half a byte a value
(``tv_mx4_save`` of ``include/tvprox.h``); ``tv_linear4`` is ``act(x W^T + b) + residual`` with x and W in that form, on the
matrix instructions that take it (``tv_linear4_fwd``).  ``TVLinear4`` is the module, made from a ``TVLinear``.  Results are
float32 or bfloat16; CUDA tensors only: there is no CPU path, and there are no gradients.
"""
from __future__ import annotations

import functools

import torch

from . import binding as _b
from .linear import _ACTS, _DTYPES, _address, _as_rows, _check, _check_tensor, _on_device, _tangent_among


def _groups(n: int) -> int:
    return -(-n // _b.TV_MX4_GROUP)


def _layout(rows: int, n: int):
    """Shapes of codes and scale bytes."""
    return (rows, 64 * _groups(n)), (_groups(n), -(-rows // 4) * 4, 4)


class Quantized4:
    """A tensor of `shape` in 4 bits, its rows (of the last axis) in groups of 128 values: `codes` uint8 [rows, 64 groups], two
    values a byte, `exps` uint8 [groups, rows up to a multiple of four, 4], a scale byte for each block of 32 (see ``tv_mx4_save``
    in ``include/tvprox.h``); `dtype` is what it is restored to."""

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor, shape, dtype: torch.dtype):
        if codes.dtype != torch.uint8 or exps.dtype != torch.uint8 or dtype not in _DTYPES:
            raise TypeError("Quantized4: uint8 codes and scale bytes and a float32 or bfloat16 dtype expected")
        if type(shape) is not torch.Size:
            shape = torch.Size(shape)
        if len(shape) < 1 or shape[-1] < 1:
            raise ValueError("Quantized4: a last axis of at least one value expected")
        want = _layout(shape.numel() // shape[-1], shape[-1])
        if (codes.shape, exps.shape) != want:
            raise ValueError("Quantized4: codes and scale bytes of shapes %r and %r expected, got %r and %r"
                             % (*want, tuple(codes.shape), tuple(exps.shape)))
        if not codes.is_cuda or exps.device != codes.device:
            raise RuntimeError("Quantized4: runs on the GPU only, codes and scale bytes on one device")
        self.codes, self.exps, self.shape, self.dtype = _on_16(codes), _on_16(exps), shape, dtype

    @classmethod
    def _saved(cls, codes, exps, shape, dtype):
        """Of what the library has just written, which needs no looking over."""
        made = cls.__new__(cls)
        made.codes, made.exps, made.shape, made.dtype = codes, exps, shape, dtype
        return made

    @property
    def device(self):
        return self.codes.device

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()

    def restore(self) -> torch.Tensor:
        """The values that the codes stand for."""
        return _restore4(self.codes, self.exps, self.shape, self.dtype)


def _on_16(t):
    """t dense and on a 16-byte boundary, as the kernels read it."""
    if not t.is_contiguous():
        t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _rows(t):
    """(t, row stride) as the kernels read it: not as a view that stands for its memory's negative."""
    return _as_rows(t.resolve_neg() if t.is_neg() else t)


@_on_device
def _restore4(codes, exps, shape, dtype):
    n = shape[-1]
    x = codes.new_empty(shape, dtype=dtype)
    _check(_b.lib().tv_mx4_load(codes.data_ptr(), exps.data_ptr(), x.data_ptr(), codes.shape[0], n, n, _DTYPES[dtype], _b._stream(None)))
    return x


@_on_device
def _save4(x, ld):
    n = x.shape[-1]
    rows = x.numel() // n
    codes, exps = _layout(rows, n)
    codes, exps = x.new_empty(codes, dtype=torch.uint8), x.new_empty(exps, dtype=torch.uint8)
    _check(_b.lib().tv_mx4_save(x.data_ptr(), codes.data_ptr(), exps.data_ptr(), rows, n, ld, _DTYPES[x.dtype], _b._stream(None)))
    return codes, exps


def tv_quantize4(x: torch.Tensor) -> Quantized4:
    """x in 4 bits, in blocks of 32 values of its last axis."""
    _check_tensor(x, "tv_quantize4")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("tv_quantize4: a last axis of at least one value expected")
    codes, exps = _save4(*_rows(x.detach()))
    return Quantized4._saved(codes, exps, x.shape, x.dtype)


@functools.lru_cache(maxsize=4096)
def _linear_desc(codes, *fields):
    desc = _b.tv_linear_desc(*fields)
    return desc, _b.tv_linear4_workspace_bytes(desc, codes)


@_on_device
def _linear4(x, x_exps, ldx, lead, weight, bias, residual, act, dtype):
    n, k = weight.shape
    y = x.new_empty((*lead, n), dtype=dtype)
    ldr = n
    if residual is not None:
        residual, ldr = _rows(residual)
    desc, nbytes = _linear_desc(x_exps is not None, lead.numel(), k, n, ldx, k, ldr, n, _DTYPES[dtype], _ACTS[act])
    ws = x.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _check(_b.lib().tv_linear4_fwd(x.data_ptr(), _address(x_exps), weight.codes.data_ptr(), weight.exps.data_ptr(), _address(bias),
                                   _address(residual), y.data_ptr(), desc, _address(ws), nbytes, _b._stream(None)))
    return y


def tv_linear4(x, weight: Quantized4, bias: torch.Tensor | None = None, residual: torch.Tensor | None = None,
               act: str = "none") -> torch.Tensor:
    """``act(x @ weight.T + bias) + residual`` over the last axis of x, with x and weight in 4 bits.

    x [..., k]: a tensor, which is taken to 4 bits in the call as ``tv_quantize4`` does it, or a Quantized4; weight [n, k];
    bias [n] and residual [..., n] of x's dtype, which is the result's; act as in ``tv_linear``.  There are no gradients.
    """
    what = "tv_linear4"
    if not isinstance(weight, Quantized4):
        raise TypeError("tv_linear4: a Quantized4 weight expected, got %s" % type(weight).__name__)
    if act not in _ACTS:
        raise ValueError("tv_linear4: act must be one of %s, got %r" % (", ".join(sorted(_ACTS)), act))
    codes = isinstance(x, Quantized4)
    if not codes and (not x.is_cuda or x.dtype not in _DTYPES):
        _check_tensor(x, what)
    if len(weight.shape) != 2 or 0 in weight.shape or len(x.shape) < 1 or x.shape[-1] != weight.shape[1]:
        raise ValueError("tv_linear4: x [..., k] and weight [n, k] expected, got %r and %r" % (tuple(x.shape), tuple(weight.shape)))
    if weight.device != x.device:
        raise TypeError("tv_linear4 (weight): one on %s expected, got one on %s" % (x.device, weight.device))
    n, lead = weight.shape[0], x.shape[:-1]
    grad = not codes and x.requires_grad
    for t, shape, name in ((bias, (n,), "bias"), (residual, (*lead, n), "residual")):
        if t is None:
            continue
        if t.dtype is not x.dtype or t.device != x.device:
            _check_tensor(t, "tv_linear4 (%s)" % name)
            raise TypeError("tv_linear4 (%s): %s on %s expected, got %s on %s" % (name, x.dtype, x.device, t.dtype, t.device))
        if t.shape != shape:
            raise ValueError("tv_linear4: %s of shape %r expected, got %r" % (name, shape, tuple(t.shape)))
        grad = grad or t.requires_grad
    if (grad and torch.is_grad_enabled()) or _tangent_among(None if codes else x, bias, residual):
        raise RuntimeError("tv_linear4: products in 4 bits have no gradients; call it under torch.no_grad() or detach its inputs")
    if bias is not None and not (bias.is_contiguous() and not bias.is_neg()):
        bias = bias.resolve_neg().contiguous()
    if codes:
        return _linear4(x.codes, x.exps, x.shape[-1], lead, weight, bias, residual, act, x.dtype)
    rows, ldx = _rows(x)
    return _linear4(rows, None, ldx, lead, weight, bias, residual, act, x.dtype)


class TVLinear4(torch.nn.Module):
    """A ``TVLinear`` for serving: its weight in 4 bits (buffers `codes` and `exps`), its bias as it was."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True, act: str = "none", device=None, dtype=None):
        super().__init__()
        if in_features < 1 or out_features < 1:
            raise ValueError("TVLinear4: sizes of at least one expected")
        if act not in _ACTS:
            raise ValueError("TVLinear4: unknown act %r" % (act,))
        self.in_features, self.out_features, self.act = in_features, out_features, act
        codes, exps = _layout(out_features, in_features)
        self.register_buffer("codes", torch.zeros(codes, dtype=torch.uint8, device=device))
        self.register_buffer("exps", torch.full(exps, 127, dtype=torch.uint8, device=device))
        self.register_buffer("bias", torch.zeros(out_features, device=device, dtype=dtype) if bias else None)

    @classmethod
    def from_linear(cls, linear) -> "TVLinear4":
        """Of a ``TVLinear``, whose weight it holds in 4 bits and whose bias it shares no memory with."""
        weight, bias = linear.weight.detach(), linear.bias
        held = tv_quantize4(weight)
        made = cls(weight.shape[1], weight.shape[0], bias is not None, linear.act, weight.device, weight.dtype)
        made.codes, made.exps = held.codes, held.exps
        if bias is not None:
            made.bias = bias.detach().clone()
        return made.train(linear.training)

    def forward(self, x, residual: torch.Tensor | None = None) -> torch.Tensor:
        weight = Quantized4(self.codes, self.exps, (self.out_features, self.in_features), x.dtype)
        return tv_linear4(x, weight, self.bias, residual, self.act)

    def extra_repr(self) -> str:
        return "%d, %d, bias=%s, act=%s" % (self.in_features, self.out_features, self.bias is not None, self.act)
