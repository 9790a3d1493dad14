"""Channel products beside the TV layer, and 8-bit checkpoints of the activations their backward pass needs.

``tv_linear`` is ``act(x W^T + b) + residual`` over the last axis of ``x`` (the mixing of channels between two TV
passes: tokens or pixels are rows), forward and backward by the library's kernels (``tv_linear_fwd`` /
``tv_linear_bwd`` of ``include/tvprox.h``).  With ``checkpoint="8bit"`` the backward pass reads ``x``, and for gelu
and silu the pre-activation, from 8-bit codes: a bit over one byte a value instead of two or four.
``tv_checkpoint8`` makes such a checkpoint of any tensor.  ``TVLinear`` is the module, ``TVMixer`` a residual block of
a TV pass along the tokens and two channel products.  float32 and bfloat16, CUDA tensors only: there is no CPU path.
"""
from __future__ import annotations

import functools
import math

import torch
from torch.autograd import forward_ad as _forward_ad

from . import binding as _b
from .layer import tv_prox_1d

_DTYPES = {torch.float32: _b.TV_F32, torch.bfloat16: _b.TV_BF16}
_ACTS = {"none": _b.TV_ACT_NONE, "relu": _b.TV_ACT_RELU, "gelu": _b.TV_ACT_GELU, "silu": _b.TV_ACT_SILU}
_CHECKPOINTS = ("full", "8bit")
_HELD_BY_DTYPE = {torch.int32: _b.TV_HELD_BITS, torch.int8: _b.TV_HELD_8BIT}
_NOTHING_HELD = _b.tv_held(None, None, _b.TV_HELD_NONE)


def _check_tensor(t: torch.Tensor, what: str, like: torch.Tensor | None = None) -> torch.Tensor:
    if not t.is_cuda:
        raise RuntimeError("%s: runs on the GPU only (got a %s tensor)" % (what, t.device))
    if t.dtype not in _DTYPES:
        raise TypeError("%s: float32 or bfloat16 expected, got %s" % (what, t.dtype))
    if like is not None and (t.dtype != like.dtype or t.device != like.device):
        raise TypeError("%s: %s on %s expected, got %s on %s" % (what, like.dtype, like.device, t.dtype, t.device))
    return t


def _as_rows(t: torch.Tensor):
    """(tensor, row stride) of t as rows of its last axis: a matrix whose rows are dense stays where it is, anything
    else is made contiguous (and with it a view that stands for its memory's negative, as the imaginary part of a conjugate,
    and rows further apart than the library takes)."""
    n = t.shape[-1]
    if t.is_contiguous():
        return t, n
    if t.dim() == 2 and (t.stride(1) == 1 or n == 1) and (n <= t.stride(0) < 1 << 31 or t.shape[0] == 1) and not t.is_neg():
        return t, (t.stride(0) if t.shape[0] > 1 else n)
    return t.contiguous(), n


def _tangent_among(*tensors) -> bool:
    """Whether forward-mode differentiation has given one of them a tangent, which the kernels would not see.  (A level
    that is not open is told by one look at its number.)"""
    return (getattr(_forward_ad, "_current_level", 0) >= 0
            and any(t is not None and _forward_ad.unpack_dual(t).tangent is not None for t in tensors))


def _blocks(n: int) -> int:
    return -(-n // _b.TV_CKPT8_BLOCK)


# A call's descriptor and workspace size, which sizes, strides, dtype, and where the operands lie between 16-byte boundaries
# say in full.
@functools.lru_cache(maxsize=4096)
def _fwd_desc(x_at, w_at, *fields):
    desc = _b.tv_linear_desc(*fields)
    return desc, _b.tv_linear_fwd_workspace_bytes_at(x_at, w_at, desc)


@functools.lru_cache(maxsize=4096)
def _bwd_desc(g_at, x_at, x_is_8bit, w_at, dx, dw, db, *fields):
    desc = _b.tv_linear_desc(*fields)
    there = [16 if t else None for t in (x_is_8bit, dx, dw, db)]
    return desc, _b.tv_linear_bwd_workspace_bytes_at(g_at, x_at, there[0], w_at, *there[1:], desc)


def _place(address):
    """A small address that lies between 16-byte boundaries as this one does."""
    return 16 + address % 16


def _on_device(call):
    """`call` with its first argument's device as the current one: that device's stream is the one it uses."""
    @functools.wraps(call)
    def wrapped(t, *rest):
        if t.get_device() == torch.cuda.current_device():
            return call(t, *rest)
        with torch.cuda.device(t.device):
            return call(t, *rest)
    return wrapped


def _address(t):
    return None if t is None else t.data_ptr()


def _check(status):
    if status:
        raise _b.TVError(status)


class Checkpoint8:
    """A tensor held in 8 bits: `codes` int8 of the tensor's shape, `exps` uint8 [rows, ceil(n / 32)], a step byte
    for each block of 32 values of a row of the last axis (see ``tv_ckpt8_save`` in ``include/tvprox.h``)."""

    def __init__(self, codes: torch.Tensor, exps: torch.Tensor, dtype: torch.dtype):
        if codes.dtype != torch.int8 or exps.dtype != torch.uint8 or dtype not in _DTYPES:
            raise TypeError("Checkpoint8: int8 codes, uint8 exponents and a float32 or bfloat16 dtype expected")
        if codes.dim() < 1 or codes.shape[-1] < 1:
            raise ValueError("Checkpoint8: a last axis of at least one value expected")
        rows = codes.numel() // codes.shape[-1]
        if tuple(exps.shape) != (rows, _blocks(codes.shape[-1])):
            raise ValueError("Checkpoint8: exponents of shape %r expected, got %r"
                             % ((rows, _blocks(codes.shape[-1])), tuple(exps.shape)))
        if not codes.is_cuda or exps.device != codes.device:
            raise RuntimeError("Checkpoint8: runs on the GPU only, codes and exponents on one device")
        self.codes, self.exps, self.dtype = codes.contiguous(), exps.contiguous(), dtype

    @classmethod
    def _saved(cls, codes, exps, dtype):
        """Of what the library has just written, which needs no looking over."""
        made = cls.__new__(cls)
        made.codes, made.exps, made.dtype = codes, exps, dtype
        return made

    @property
    def shape(self):
        return self.codes.shape

    @property
    def nbytes(self) -> int:
        return self.codes.numel() + self.exps.numel()

    def restore(self) -> torch.Tensor:
        """The values that the codes stand for."""
        return _restore8(self.codes, self.exps, self.dtype)


@_on_device
def _restore8(codes, exps, dtype):
    n = codes.shape[-1]
    x = codes.new_empty(codes.shape, dtype=dtype)
    _check(_b.lib().tv_ckpt8_load(codes.data_ptr(), exps.data_ptr(), x.data_ptr(), exps.shape[0], n, n, _DTYPES[dtype], _b._stream(None)))
    return x


@_on_device
def _save8(x, ld):
    """(codes, exponents) of x as rows (see _as_rows)."""
    n = x.shape[-1]
    rows = x.numel() // n
    codes = x.new_empty(x.shape, dtype=torch.int8)
    exps = x.new_empty((rows, _blocks(n)), dtype=torch.uint8)
    _check(_b.lib().tv_ckpt8_save(x.data_ptr(), codes.data_ptr(), exps.data_ptr(), rows, n, ld, _DTYPES[x.dtype], _b._stream(None)))
    return codes, exps


def tv_checkpoint8(x: torch.Tensor) -> Checkpoint8:
    """An 8-bit checkpoint of x, in blocks of 32 values of its last axis."""
    _check_tensor(x, "tv_checkpoint8")
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError("tv_checkpoint8: a last axis of at least one value expected")
    codes, exps = _save8(*_as_rows(x.detach()))
    return Checkpoint8._saved(codes, exps, x.dtype)


@_on_device
def _forward(x, ldx, weight, ldw, bias, residual, act, hold):
    """(y, what is held of z, its exponents): x and weight as rows, hold one of None, "full", "8bit"."""
    k, n, code, dtype = x.shape[-1], weight.shape[0], _ACTS[act], _DTYPES[x.dtype]
    m = x.numel() // k
    y = x.new_empty((*x.shape[:-1], n))
    ldr = n
    if residual is not None:
        residual, ldr = _as_rows(residual)
    data = exps = None
    held = _NOTHING_HELD
    if hold is not None and code != _b.TV_ACT_NONE:
        if code == _b.TV_ACT_RELU:
            data, kind = x.new_empty((m, _blocks(n)), dtype=torch.int32), _b.TV_HELD_BITS
        elif hold == "8bit":
            data, kind = x.new_empty((m, n), dtype=torch.int8), _b.TV_HELD_8BIT
            exps = x.new_empty((m, _blocks(n)), dtype=torch.uint8)
        else:
            data, kind = x.new_empty((m, n)), _b.TV_HELD_PLAIN
        held = _b.tv_held(data.data_ptr(), _address(exps), kind)
    at_x, at_w = x.data_ptr(), weight.data_ptr()
    desc, nbytes = _fwd_desc(_place(at_x), _place(at_w), m, k, n, ldx, ldw, ldr, n, dtype, code)
    ws = x.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _check(_b.lib().tv_linear_fwd(at_x, at_w, _address(bias), _address(residual), y.data_ptr(), held, desc,
                                  _address(ws), nbytes, _b._stream(None)))
    return y, data, exps


@_on_device
def _backward(g, x, x_exps, ldx, data, exps, weight, ldw, act, want):
    """(dx, dw, db), None where not wanted.  x: rows, or the codes of its checkpoint (x_exps given)."""
    n, k = weight.shape
    m = g.numel() // n
    code, dtype = _ACTS[act], _DTYPES[g.dtype]
    g, ldg = _as_rows(g)
    kind = _b.TV_HELD_NONE
    if data is not None:
        kind = _HELD_BY_DTYPE.get(data.dtype, _b.TV_HELD_PLAIN)
    dx = g.new_empty((*g.shape[:-1], k)) if want[0] else None
    dw = g.new_empty((n, k)) if want[1] else None
    db = g.new_empty(n) if want[2] else None
    at_g, at_x, at_w = g.data_ptr(), _address(x), weight.data_ptr()
    desc, nbytes = _bwd_desc(_place(at_g), _place(at_x or 0), x_exps is not None, _place(at_w), *want, m, k, n, ldx, ldw, n, ldg, dtype, code)
    ws = g.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _check(_b.lib().tv_linear_bwd(at_g, at_x, _address(x_exps), _b.tv_held(_address(data), _address(exps), kind),
                                  at_w, _address(dx), _address(dw), _address(db),
                                  desc, _address(ws), nbytes, _b._stream(None)))
    return dx, dw, db


class _Linear(torch.autograd.Function):
    """y = act(x W^T + b) + r; x and weight come as rows (see _as_rows)."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, act, checkpoint):
        rows, ldx = _as_rows(x)
        wrows, ldw = _as_rows(weight)
        # (z is for the slopes, which the residual's gradient does without)
        hold = checkpoint if any(ctx.needs_input_grad[:3]) else None
        y, data, exps = _forward(rows, ldx, wrows, ldw, bias, residual, act, hold)
        x_exps = None
        if not ctx.needs_input_grad[1]:
            rows = None                            # only dW reads x
        elif checkpoint == "8bit":
            rows, x_exps = _save8(rows, ldx)
        saved = (rows, x_exps, data, exps, wrows)
        ctx.save_for_backward(*saved)
        ctx.saved_as = [None if t is None else (t.shape, t.dtype) for t in saved]
        ctx.act, ctx.has_bias = act, bias is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        if _tangent_among(g):
            raise NotImplementedError("tv_linear: the gradients have no forward-mode derivative")
        # (hooks on saved tensors may bring back others, with the same values in strides of their own)
        saved, where = ctx.saved_tensors, g.get_device()
        for t, was in zip(saved, ctx.saved_as):
            if t is not None and (t.dtype is not was[1] or t.shape != was[0] or t.get_device() != where or t.is_meta):
                raise RuntimeError("tv_linear: a hook on saved tensors has brought back one of another shape, type or device")
        x, x_exps, data, exps, weight = saved
        need = ctx.needs_input_grad
        want = (need[0], need[1], ctx.has_bias and need[2])
        dx = dw = db = None
        if any(want):
            if x_exps is not None:
                x, x_exps = x.contiguous(), x_exps.contiguous()
            if data is not None:
                data = data.contiguous()
            if exps is not None:
                exps = exps.contiguous()
            weight, ldw = _as_rows(weight)
            x, ldx = (None, ldw) if x is None else _as_rows(x)
            dx, dw, db = _backward(g, x, x_exps, ldx, data, exps, weight, ldw, ctx.act, want)
        return dx, dw, db, (g if need[3] else None), None, None


def _check_linear(x, weight, act, what):
    if act not in _ACTS:
        raise ValueError("%s: act must be one of %s, got %r" % (what, ", ".join(sorted(_ACTS)), act))
    if weight.dim() != 2 or x.dim() < 1 or x.shape[-1] != weight.shape[1] or 0 in weight.shape:
        raise ValueError("%s: x [..., k] and weight [n, k] expected, got %r and %r"
                         % (what, tuple(x.shape), tuple(weight.shape)))


def tv_linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None,
              residual: torch.Tensor | None = None, act: str = "none", checkpoint: str = "full") -> torch.Tensor:
    """Differentiable ``act(x @ weight.T + bias) + residual`` over the last axis of x.

    x [..., k], weight [n, k], bias [n], residual [..., n], all of one dtype (float32 or bfloat16); act "none",
    "relu", "gelu" (with erf) or "silu".  checkpoint: what is kept for the backward pass, "full" (x and the
    pre-activation as they are) or "8bit" (both in 8-bit codes; ReLU keeps a bit a value either way).
    """
    if not (x.is_cuda and weight.is_cuda and x.dtype in _DTYPES and weight.dtype is x.dtype and weight.get_device() == x.get_device()):
        _check_tensor(x, "tv_linear")
        _check_tensor(weight, "tv_linear (weight)", x)
    _check_linear(x, weight, act, "tv_linear")
    if checkpoint not in _CHECKPOINTS:
        raise ValueError("tv_linear: checkpoint must be one of %s, got %r" % (", ".join(_CHECKPOINTS), checkpoint))
    n = weight.shape[0]
    if bias is not None:
        _check_tensor(bias, "tv_linear (bias)", x)
        if bias.dim() != 1 or bias.shape[0] != n:
            raise ValueError("tv_linear: bias of shape (%d,) expected, got %r" % (n, tuple(bias.shape)))
        bias = bias.contiguous()
    if residual is not None:
        _check_tensor(residual, "tv_linear (residual)", x)
        if residual.shape != (*x.shape[:-1], n):
            raise ValueError("tv_linear: residual of shape %r expected, got %r" % ((*x.shape[:-1], n), tuple(residual.shape)))
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or (bias is not None and bias.requires_grad)
                                    or (residual is not None and residual.requires_grad)) \
            or _tangent_among(x, weight, bias, residual):              # (which apply refuses)
        return _Linear.apply(x, weight, bias, residual, act, checkpoint)
    x, ldx = _as_rows(x)
    weight, ldw = _as_rows(weight)
    return _forward(x, ldx, weight, ldw, bias, residual, act, None)[0]


def tv_linear_backward(g: torch.Tensor, x, z, weight: torch.Tensor, act: str = "none", bias_grad: bool = False,
                       input_grad: bool = True, weight_grad: bool = True):
    """(dx, dw, db) of ``tv_linear`` from what a program holds itself: x the input or its Checkpoint8; z the
    pre-activation or its Checkpoint8 (gelu, silu), the int32 words of its signs (relu: bit j % 32 of word j / 32 of a
    row set where not z <= 0) or None (none).  db is None unless bias_grad; input_grad and weight_grad say whether dx and dW
    are wanted (None otherwise)."""
    _check_tensor(g, "tv_linear_backward")
    _check_tensor(weight, "tv_linear_backward (weight)", g)
    n = weight.shape[0] if weight.dim() == 2 else -1
    _check_linear(x.codes if isinstance(x, Checkpoint8) else x, weight, act, "tv_linear_backward")
    if tuple(g.shape) != tuple(x.shape[:-1]) + (n,):
        raise ValueError("tv_linear_backward: g of shape %r expected, got %r" % (tuple(x.shape[:-1]) + (n,), tuple(g.shape)))
    m = g.numel() // n
    x_exps = None
    if _tangent_among(g, weight, *(t for t in (x, z) if isinstance(t, torch.Tensor))):
        raise NotImplementedError("tv_linear_backward: the gradients have no forward-mode derivative")
    if isinstance(x, Checkpoint8):
        x, x_exps, ldx = x.codes, x.exps, x.shape[-1]
        if x.device != g.device:
            raise TypeError("tv_linear_backward (x): a checkpoint on %s expected, got one on %s" % (g.device, x.device))
    else:
        _check_tensor(x, "tv_linear_backward (x)", g)
        x, ldx = _as_rows(x)
    data = exps = None
    if act == "none":
        if z is not None:
            raise ValueError("tv_linear_backward: nothing of z is held without an activation")
    elif act == "relu":
        if not isinstance(z, torch.Tensor) or z.dtype != torch.int32 or tuple(z.shape) != (m, _blocks(n)) or z.device != g.device:
            raise ValueError("tv_linear_backward: relu takes int32 sign words of shape %r" % ((m, _blocks(n)),))
        data = z.contiguous()
    elif isinstance(z, Checkpoint8):
        if z.codes.numel() != m * n or z.shape[-1] != n or z.codes.device != g.device:
            raise ValueError("tv_linear_backward: z of %d rows of %d values expected, got %r" % (m, n, tuple(z.shape)))
        data, exps = z.codes, z.exps
    else:
        if not isinstance(z, torch.Tensor) or z.shape != g.shape:
            raise ValueError("tv_linear_backward: z of g's shape, or its Checkpoint8, expected")
        data = _check_tensor(z, "tv_linear_backward (z)", g).contiguous()
    wrows, ldw = _as_rows(weight)
    want = (bool(input_grad), bool(weight_grad), bool(bias_grad))
    if not any(want):
        return None, None, None
    return _backward(g, x, x_exps, ldx, data, exps, wrows, ldw, act, want)


class TVLinear(torch.nn.Module):
    """``tv_linear`` with its weight [out_features, in_features] and bias as parameters."""

    def __init__(self, in_features: int, out_features: int, bias: bool = True, act: str = "none",
                 checkpoint: str = "full", device=None, dtype=None):
        super().__init__()
        if in_features < 1 or out_features < 1:
            raise ValueError("TVLinear: sizes of at least one expected")
        if act not in _ACTS or checkpoint not in _CHECKPOINTS:
            raise ValueError("TVLinear: unknown act %r or checkpoint %r" % (act, checkpoint))
        self.act, self.checkpoint = act, checkpoint
        like = dict(device=device, dtype=dtype)
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, **like))
        self.bias = torch.nn.Parameter(torch.empty(out_features, **like)) if bias else None
        bound = 1.0 / math.sqrt(in_features)
        torch.nn.init.uniform_(self.weight, -bound, bound)
        if bias:
            torch.nn.init.uniform_(self.bias, -bound, bound)

    def forward(self, x: torch.Tensor, residual: torch.Tensor | None = None) -> torch.Tensor:
        return tv_linear(x, self.weight, self.bias, residual, self.act, self.checkpoint)

    def extra_repr(self) -> str:
        return "%d, %d, bias=%s, act=%s, checkpoint=%s" % (self.weight.shape[1], self.weight.shape[0],
                                                           self.bias is not None, self.act, self.checkpoint)


class TVMixer(torch.nn.Module):
    """Residual block over tokens [B, T, C]: a TV pass along T (1D operator, a trainable lambda a channel through a
    SoftPlus), then two channel products:  x + W2 act(W1 tv(x) + b1) + b2.

    The TV pass runs in fp32 (its rows lie along the second axis, for which the library has no bf16 storage); the
    products run in the block's dtype and keep their activations as `checkpoint` says.
    """

    def __init__(self, channels: int, hidden: int, act: str = "gelu", checkpoint: str = "8bit",
                 init_lambda: float = 0.05, device=None, dtype=None):
        super().__init__()
        if init_lambda <= 0.0:
            raise ValueError("TVMixer: init_lambda must be positive")
        raw = init_lambda + math.log(-math.expm1(-init_lambda))              # inverse of the SoftPlus
        self.raw_lambda = torch.nn.Parameter(torch.full((channels,), raw, dtype=torch.float32, device=device))
        like = dict(checkpoint=checkpoint, device=device, dtype=dtype)
        self.expand = TVLinear(channels, hidden, act=act, **like)
        self.reduce = TVLinear(hidden, channels, **like)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if x.dim() != 3 or x.shape[-1] != self.raw_lambda.numel():
            raise ValueError("TVMixer: [B, T, %d] expected, got %r" % (self.raw_lambda.numel(), tuple(x.shape)))
        lam = torch.nn.functional.softplus(self.raw_lambda)
        smooth = tv_prox_1d(x.float(), lam, axis=1).to(x.dtype)
        return self.reduce(self.expand(smooth), residual=x)
