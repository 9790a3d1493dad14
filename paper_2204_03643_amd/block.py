"""The borders of residual blocks (norms before and after a block, gate, scale, dropout, residual) and dropout by itself.

``tv_norm`` is the norm before a block, ``tv_residual`` what follows it, ``x + dropout(scale * act(gate) * norm(f))`` and,
on request, the norm before the next block of the sum; one pass over the rows each way, by the library's kernels
(``tv_block_fwd`` / ``tv_block_bwd`` of ``include/tvprox.h``).  ``tv_dropout`` takes its numbers from a counter-based
generator: no mask is stored, and the same seed and offset always mean the same mask.  ``TVNorm`` and ``TVResidual`` are the
modules.  float32 and bfloat16, CUDA tensors only: there is no CPU path.

A step that is captured into a graph starts from leaves of which no eager step's graph is alive any more: torch's engine would
otherwise wait for the eager step's stream within the capture.
"""
from __future__ import annotations

import functools
import math
import typing

import torch

from . import binding as _b
from .linear import _DTYPES, _address, _as_rows, _check, _check_tensor, _on_device, _tangent_among

_NORMS = {"none": _b.TV_NORM_NONE, "rms": _b.TV_NORM_RMS, "layer": _b.TV_NORM_LAYER}
_GATE_ACTS = {"none": _b.TV_GATE_PLAIN, "sigmoid": _b.TV_GATE_SIGMOID, "silu": _b.TV_GATE_SILU}
_NO_DROP = _b.tv_drop(0, 0, None, 0)


def _once_differentiable(backward):
    """torch's decorator where a graph of the gradients is asked for (which refuses to differentiate it); without one the
    function itself, which saves what the decorator costs in every step."""
    refusing = torch.autograd.function.once_differentiable(backward)

    @functools.wraps(backward)
    def call(ctx, *grads):
        return refusing(ctx, *grads) if torch.is_grad_enabled() else backward(ctx, *grads)
    return call


class _Border(typing.NamedTuple):
    """What a border does, beside its tensors."""
    norm: int
    next_norm: int
    act: int
    eps: float
    gate_div: int
    drop: int                # of 65536
    offset: int


_border = functools.lru_cache(maxsize=4096)(_Border)


def _check_number(v, what):
    if isinstance(v, bool) or not isinstance(v, int):
        raise TypeError("%s: a whole number expected, got %r" % (what, v))
    if not -(1 << 63) <= v < 1 << 64:
        raise ValueError("%s: a number of 64 bits expected, got %r" % (what, v))
    return v & 0xFFFFFFFFFFFFFFFF


def _check_drop(p, seed, offset, like, what):
    """(p in 1/65536, seed, seed tensor, offset)"""
    if not 0.0 <= p <= 1.0:
        raise ValueError("%s: a probability between 0 and 1 expected, got %r" % (what, p))
    drop = int(math.floor(65536.0 * p + 0.5))
    if not drop:
        return 0, 0, None, 0
    at = None
    if isinstance(seed, torch.Tensor):
        if seed.dtype is not torch.int64 or seed.numel() != 1 or seed.device != like.device:
            raise TypeError("%s: a seed tensor of one int64 on %s expected, got %r of %s on %s"
                            % (what, like.device, tuple(seed.shape), seed.dtype, seed.device))
        at, seed = seed.detach(), 0
    elif seed is None:
        raise ValueError("%s: dropout needs a seed" % what)
    return drop, _check_number(seed, what + " (seed)"), at, _check_number(offset, what + " (offset)")


def _check_channels(t, n, what, like):
    if t is None:
        return None
    if t.dtype is not like.dtype or t.get_device() != like.get_device():
        _check_tensor(t, what, like)
    if t.numel() != n or t.dim() != 1:
        raise ValueError("%s: shape (%d,) expected, got %r" % (what, n, tuple(t.shape)))
    return _dense(t)


def _dense(t):
    """t without gaps, and not as a view that stands for its memory's negative."""
    return t if t.is_contiguous() and not t.is_neg() else t.resolve_neg().contiguous()


def _rows(t):
    return _as_rows(t.resolve_neg() if t.is_neg() else t)


def _gate_div(x, gate, what):
    """How many rows of x share a row of the gate: x's shape, with ones in its last leading axes where they do."""
    if gate.shape == x.shape:
        return 1
    lead = tuple(x.shape[:-1])
    rows = tuple(gate.shape[:-1]) if gate.dim() > 1 or x.dim() == 1 else (1,) * len(lead)
    k = len(rows)
    while k and rows[k - 1] == 1:
        k -= 1
    if gate.dim() < 1 or gate.shape[-1] != x.shape[-1] or len(rows) != len(lead) or rows[:k] != lead[:k]:
        raise ValueError("%s: a gate of x's shape %r, or with ones in its last leading axes, expected, got %r"
                         % (what, tuple(x.shape), tuple(gate.shape)))
    return max(1, math.prod(lead[k:]))


# How much workspace a backward call needs, which its sizes, whether there is an f, a bias and a gate, and what is wanted say in
# full (a bias adds a sum over the rows to dscale's).
@functools.lru_cache(maxsize=4096)
def _workspace_bytes(m, n, dtype, has_f, has_bias, has_gate, border, want):
    ins = _b.tv_block_in(16, 16 if has_f else None, None, 16 if has_bias else None, 16 if has_gate else None, None, None, None)
    dx, df, dweight, dbias, dgate, dscale, dnext_weight, dnext_bias = (16 if w else None for w in want)
    return _b.tv_block_bwd_workspace_bytes(ins, _b.tv_block_grads(dx, df, dgate, dweight, dbias, dscale, dnext_weight, dnext_bias),
                                           _desc(m, n, n, n, n, dtype, border))


@functools.lru_cache(maxsize=4096)
def _desc(m, n, ldx, ldf, ldg, dtype, border, remake_y=0):
    return _b.tv_block_desc(m, n, ldx, ldf, ldg, border.gate_div, dtype, border.norm, border.next_norm, border.act, border.eps,
                            _NO_DROP, remake_y)


def _desc_of(m, n, ldx, ldf, ldg, dtype, border, seed, seed_at, remake_y=0):
    if not border.drop:
        return _desc(m, n, ldx, ldf, ldg, dtype, border, remake_y)
    return _b.tv_block_desc(m, n, ldx, ldf, ldg, border.gate_div, dtype, border.norm, border.next_norm, border.act, border.eps,
                            _b.tv_drop(seed, border.offset, _address(seed_at), border.drop), remake_y)


def _remakes_y(dtype):
    """Whether the next norm's gradient makes y again of x and f: where y was rounded when it was returned."""
    return int(dtype is torch.bfloat16)


@_on_device
def _forward(x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at, hold):
    """(y, h, stats): None where there is none."""
    n = x.shape[-1]
    m = x.numel() // n
    rows, ldx = _rows(x)
    h = stats = at_gate = at_h = at_stats = None
    ldg = n
    frows, ldf = _rows(f)
    y = x.new_empty(x.shape)
    if gate is not None:
        grows, ldg = _rows(gate)
        at_gate = grows.data_ptr()
    if border.next_norm:
        h = x.new_empty(x.shape)
        at_h = h.data_ptr()
    if hold:
        stats = x.new_empty((m, 4), dtype=torch.float32)
        at_stats = stats.data_ptr()
    ins = _b.tv_block_in(rows.data_ptr(), frows.data_ptr(), _address(weight), _address(bias), at_gate, _address(scale),
                         _address(next_weight), _address(next_bias))
    _check(_b.lib().tv_block_fwd(ins, y.data_ptr(), at_h, at_stats, _desc_of(m, n, ldx, ldf, ldg, _DTYPES[x.dtype], border, seed, seed_at),
                                 _b._stream(None)))
    return y, h, stats


@_on_device
def _backward(like, dy, dh, after, f, weight, bias, gate, scale, next_weight, stats, border, seed, seed_at, want):
    """Gradients of x, f, weight, bias, gate, scale, next_weight, next_bias, None where not wanted.  after: with a next norm y,
    or x where y is made again."""
    shape, n = like.shape, like.shape[-1]
    m, dtype = like.numel() // n, _DTYPES[like.dtype]
    at_after = at_gate = None
    ldx = ldg = n
    if after is not None:
        after, ldx = _rows(after)
        at_after = after.data_ptr()
    f, ldf = _rows(f)
    if gate is not None:
        grows, ldg = _rows(gate)
        at_gate = grows.data_ptr()
    shapes = (shape, shape, n, n, None if gate is None else gate.shape, n, n, n)
    made = [like.new_empty(s) if w else None for s, w in zip(shapes, want)]
    dx, df, dweight, dbias, dgate, dscale, dnext_weight, dnext_bias = [None if t is None else t.data_ptr() for t in made]
    ins = _b.tv_block_in(at_after, f.data_ptr(), _address(weight), _address(bias), at_gate, _address(scale), _address(next_weight), None)
    nbytes = _workspace_bytes(m, n, dtype, True, bias is not None, gate is not None, border, want)
    ws = like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _check(_b.lib().tv_block_bwd(_address(dy), _address(dh), ins, _address(stats),
                                 _b.tv_block_grads(dx, df, dgate, dweight, dbias, dscale, dnext_weight, dnext_bias),
                                 _desc_of(m, n, ldx, ldf, ldg, dtype, border, seed, seed_at, _remakes_y(like.dtype)), _address(ws), nbytes, _b._stream(None)))
    return made


class _BorderFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at):
        if _tangent_among(x, f, weight, bias, gate, scale, next_weight, next_bias):
            raise NotImplementedError("tv_residual: no forward-mode derivative")
        normed = border.next_norm or border.norm
        y, h, stats = _forward(x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at, normed)
        after = (x if _remakes_y(x.dtype) else y) if border.next_norm else None
        saved = (after, f, weight, bias, gate, scale, next_weight, stats, seed_at)
        ctx.save_for_backward(*saved)
        ctx.saved_as = [None if t is None else (t.shape, t.dtype) for t in saved]
        ctx.border, ctx.seed = border, seed
        ctx.set_materialize_grads(False)
        return y if h is None else (y, h)

    @staticmethod
    @_once_differentiable
    def backward(ctx, *grads):
        border, need = ctx.border, ctx.needs_input_grad
        saved = ctx.saved_tensors
        like = next((g for g in grads if g is not None), None)
        if like is None:
            return (None,) * 11
        if _tangent_among(*grads):
            raise NotImplementedError("tv_residual: the gradients have no forward-mode derivative")
        # (hooks on saved tensors may bring back others, with the same values in strides of their own)
        for t, was in zip(saved, ctx.saved_as):
            if t is not None and (t.dtype is not was[1] or t.shape != was[0] or t.get_device() != like.get_device() or t.is_meta):
                raise RuntimeError("tv_residual: a hook on saved tensors has brought back one of another shape, type or device")
        after, f, weight, bias, gate, scale, next_weight, stats, seed_at = saved
        dy, dh = grads if border.next_norm else (grads[0], None)
        if dy is not None:
            dy = _dense(dy)
        if dh is not None:
            dh = _dense(dh)
        # without a gradient through the next norm, x's is y's
        want = (need[0] and dh is not None, *need[1:8])
        if like.numel() == 0:
            shapes = [like.shape, like.shape] + [like.shape[-1:]] * 6
            if gate is not None:
                shapes[4] = gate.shape
            made = [like.new_zeros(s) if w else None for s, w in zip(shapes, need)]
        elif any(want):
            weight, bias, scale, next_weight, stats = [None if t is None else _dense(t) for t in (weight, bias, scale, next_weight, stats)]
            made = _backward(like, dy, dh, after, f, weight, bias, gate, scale, next_weight, stats, border, ctx.seed, seed_at, want)
        else:
            made = [None] * 8
        if need[0] and dh is None:
            made[0] = dy
        return (*made, None, None, None)


@_on_device
def _norm_forward(x, weight, bias, border, hold):
    """(h, stats)"""
    n = x.shape[-1]
    m = x.numel() // n
    rows, ldx = _rows(x)
    h = x.new_empty(x.shape)
    stats = x.new_empty((m, 4), dtype=torch.float32) if hold else None
    ins = _b.tv_block_in(rows.data_ptr(), None, None, None, None, None, _address(weight), _address(bias))
    _check(_b.lib().tv_block_fwd(ins, None, h.data_ptr(), _address(stats), _desc(m, n, ldx, n, n, _DTYPES[x.dtype], border), _b._stream(None)))
    return h, stats


@_on_device
def _norm_backward(g, x, weight, stats, border, want):
    """Gradients of x, weight and bias, None where not wanted."""
    n = g.shape[-1]
    m, dtype = g.numel() // n, _DTYPES[g.dtype]
    x, ldx = _rows(x)
    dx = g.new_empty(g.shape) if want[0] else None
    dweight = g.new_empty(n) if want[1] else None
    dbias = g.new_empty(n) if want[2] else None
    ins = _b.tv_block_in(x.data_ptr(), None, None, None, None, None, _address(weight), None)
    nbytes = _workspace_bytes(m, n, dtype, False, False, False, border, (want[0], False, False, False, False, False, want[1], want[2]))
    ws = g.new_empty(nbytes, dtype=torch.uint8) if nbytes else None
    _check(_b.lib().tv_block_bwd(None, g.data_ptr(), ins, stats.data_ptr(),
                                 _b.tv_block_grads(_address(dx), None, None, None, None, None, _address(dweight), _address(dbias)),
                                 _desc(m, n, ldx, n, n, dtype, border), _address(ws), nbytes, _b._stream(None)))
    return dx, dweight, dbias


class _Norm(torch.autograd.Function):
    """A norm alone, which is called so often that it does without the border's other seven tensors."""

    @staticmethod
    def forward(ctx, x, weight, bias, border):
        if _tangent_among(x, weight, bias):
            raise NotImplementedError("tv_norm: no forward-mode derivative")
        h, stats = _norm_forward(x, weight, bias, border, True)
        saved = (x, weight, stats)
        ctx.save_for_backward(*saved)
        ctx.saved_as = [None if t is None else (t.shape, t.dtype) for t in saved]
        ctx.border = border
        return h

    @staticmethod
    @_once_differentiable
    def backward(ctx, g):
        if _tangent_among(g):
            raise NotImplementedError("tv_norm: the gradients have no forward-mode derivative")
        saved, where = ctx.saved_tensors, g.get_device()
        for t, was in zip(saved, ctx.saved_as):
            if t is not None and (t.dtype is not was[1] or t.shape != was[0] or t.get_device() != where or t.is_meta):
                raise RuntimeError("tv_norm: a hook on saved tensors has brought back one of another shape, type or device")
        x, weight, stats = saved
        need = ctx.needs_input_grad
        if g.numel() == 0:
            n = g.shape[-1]
            return (g if need[0] else None), (g.new_zeros(n) if need[1] else None), (g.new_zeros(n) if need[2] else None), None
        dx, dweight, dbias = _norm_backward(_dense(g), x, None if weight is None else _dense(weight), _dense(stats), ctx.border, need)
        return dx, dweight, dbias, None


def _check_rows(x, what):
    if not x.is_cuda or x.dtype not in _DTYPES:
        _check_tensor(x, what)
    n = x.shape[-1] if x.dim() else 0
    if n < 1:
        raise ValueError("%s: a last axis of at least one channel expected" % what)
    if n > _b.TV_MAX_LENGTH:
        raise ValueError("%s: at most %d channels, got %d" % (what, _b.TV_MAX_LENGTH, n))
    return n


def _check_eps(eps, what):
    if not 0.0 <= eps < math.inf:
        raise ValueError("%s: eps of at least 0 expected, got %r" % (what, eps))
    return float(eps)


def _apply(x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at):
    grad = torch.is_grad_enabled() and (
        x.requires_grad or f.requires_grad or (weight is not None and weight.requires_grad)
        or (bias is not None and bias.requires_grad) or (gate is not None and gate.requires_grad)
        or (scale is not None and scale.requires_grad) or (next_weight is not None and next_weight.requires_grad) or (next_bias is not None and next_bias.requires_grad))
    if grad or _tangent_among(x, f, weight, bias, gate, scale, next_weight, next_bias):
        return _BorderFunction.apply(x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at)
    y, h, _ = _forward(x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at, False)
    return y if h is None else (y, h)


def tv_norm(x: torch.Tensor, weight: torch.Tensor | None = None, bias: torch.Tensor | None = None, kind: str = "rms",
            eps: float = 1e-6) -> torch.Tensor:
    """Differentiable ``(x - mu) * r * weight + bias`` over the last axis of x, ``r = (mean((x - mu)^2) + eps)^(-1/2)``:
    mu is the mean (kind "layer") or 0 ("rms").  weight and bias [n], or None."""
    n = _check_rows(x, "tv_norm")
    if kind not in ("rms", "layer"):
        raise ValueError("tv_norm: kind must be rms or layer, got %r" % (kind,))
    weight = _check_channels(weight, n, "tv_norm (weight)", x)
    bias = _check_channels(bias, n, "tv_norm (bias)", x)
    border = _border(0, _NORMS[kind], 0, _check_eps(eps, "tv_norm"), 1, 0, 0)
    if (torch.is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad)
                                     or (bias is not None and bias.requires_grad))) or _tangent_among(x, weight, bias):
        return _Norm.apply(x, weight, bias, border)
    return _norm_forward(x, weight, bias, border, False)[0]


def tv_residual(x: torch.Tensor, f: torch.Tensor, norm: str = "none", weight: torch.Tensor | None = None,
                bias: torch.Tensor | None = None, gate: torch.Tensor | None = None, gate_act: str = "none",
                scale: torch.Tensor | None = None, dropout: float = 0.0, seed=None, offset: int = 0, next_norm: str = "none",
                next_weight: torch.Tensor | None = None, next_bias: torch.Tensor | None = None, eps: float = 1e-6):
    """Differentiable ``y = x + dropout(scale * act(gate) * norm(f))`` over the last axis; with a next norm ``(y, h)``, h the
    next norm of y (before y is rounded, in its gradients too: in bfloat16 they take y from x and f again).

    x, f [..., n]; norm and next_norm "none", "rms" or "layer" with weights and biases [n] or None (see ``tv_norm``);
    gate of x's shape, or with ones in its last leading axes (one row for all rows that share it), gate_act "none", "sigmoid" or
    "silu"; scale [n]; dropout, seed and offset as in ``tv_dropout``.  All of one dtype.
    """
    what = "tv_residual"
    n = _check_rows(x, what)
    if f.dtype is not x.dtype or f.get_device() != x.get_device():
        _check_tensor(f, "tv_residual (f)", x)
    if f.shape != x.shape:
        raise ValueError("tv_residual: f of shape %r expected, got %r" % (tuple(x.shape), tuple(f.shape)))
    if norm not in _NORMS or next_norm not in _NORMS:
        raise ValueError("tv_residual: norm and next_norm must be none, rms or layer, got %r and %r" % (norm, next_norm))
    if gate_act not in _GATE_ACTS or (gate is None and gate_act != "none"):
        raise ValueError("tv_residual: gate_act must be none, sigmoid or silu (none without a gate), got %r" % (gate_act,))
    if (norm == "none" and (weight is not None or bias is not None)) or (next_norm == "none" and (next_weight is not None or next_bias is not None)):
        raise ValueError("tv_residual: weight and bias belong to a norm")
    weight = _check_channels(weight, n, "tv_residual (weight)", x)
    bias = _check_channels(bias, n, "tv_residual (bias)", x)
    scale = _check_channels(scale, n, "tv_residual (scale)", x)
    next_weight = _check_channels(next_weight, n, "tv_residual (next_weight)", x)
    next_bias = _check_channels(next_bias, n, "tv_residual (next_bias)", x)
    div = 1
    if gate is not None:
        if gate.dtype is not x.dtype or gate.get_device() != x.get_device():
            _check_tensor(gate, "tv_residual (gate)", x)
        div = _gate_div(x, gate, what)
    drop, seed, seed_at, offset = _check_drop(dropout, seed, offset, x, what)
    border = _border(_NORMS[norm], _NORMS[next_norm], _GATE_ACTS[gate_act], _check_eps(eps, what), div, drop, offset)
    return _apply(x, f, weight, bias, gate, scale, next_weight, next_bias, border, seed, seed_at)


@_on_device
def _drop(x, how, seed_at):
    """how: (drop, seed, offset)"""
    drop, seed, offset = how
    rows, ldx = _rows(x if x.dim() else x.view(1))
    n = rows.shape[-1]
    y = x.new_empty(x.shape)
    _check(_b.lib().tv_drop_apply(rows.data_ptr(), y.data_ptr(), x.numel() // n, n, ldx, _DTYPES[x.dtype],
                                  _b.tv_drop(seed, offset, _address(seed_at), drop), _b._stream(None)))
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, how, seed_at):
        if _tangent_among(x):
            raise NotImplementedError("tv_dropout: no forward-mode derivative")
        ctx.how = how
        if seed_at is not None:
            ctx.save_for_backward(seed_at)
        return _drop(x, how, seed_at)

    @staticmethod
    @_once_differentiable
    def backward(ctx, g):
        if _tangent_among(g):
            raise NotImplementedError("tv_dropout: the gradient has no forward-mode derivative")
        saved = ctx.saved_tensors
        if saved and (saved[0].dtype is not torch.int64 or saved[0].numel() != 1 or saved[0].device != g.device):
            raise RuntimeError("tv_dropout: a hook on saved tensors has brought back one of another shape, type or device")
        return _drop(g, ctx.how, saved[0] if saved else None), None, None


def tv_dropout(x: torch.Tensor, p: float, seed, offset: int = 0) -> torch.Tensor:
    """Differentiable dropout: zero with probability p (taken to the nearest multiple of 1/65536), x / (1 - p) otherwise.

    Which values are dropped is a function of seed and offset (whole numbers of 64 bits), the row (of the last axis) and the
    column alone.  seed may be an int64 tensor of one element on x's device, which is read when the kernel runs: a captured graph
    drops others in every replay if the program changes it in between.  It must not change between a call and its backward pass;
    calls of one step are told apart by their offsets.  With p below 2^-17 the result is x itself.
    """
    _check_tensor(x, "tv_dropout")
    drop, seed, seed_at, offset = _check_drop(p, seed, offset, x, "tv_dropout")
    if not drop or x.numel() == 0:
        return x
    if (torch.is_grad_enabled() and x.requires_grad) or _tangent_among(x):
        return _Dropout.apply(x, (drop, seed, offset), seed_at)
    return _drop(x, (drop, seed, offset), seed_at)


class TVNorm(torch.nn.Module):
    """``tv_norm`` with its weight (ones) and, for layer norms, bias (zeros) [channels] as parameters."""

    def __init__(self, channels: int, kind: str = "rms", bias: bool | None = None, eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        if not 1 <= channels <= _b.TV_MAX_LENGTH:
            raise ValueError("TVNorm: 1 to %d channels expected" % _b.TV_MAX_LENGTH)
        if kind not in ("rms", "layer"):
            raise ValueError("TVNorm: kind must be rms or layer, got %r" % (kind,))
        self.kind, self.eps = kind, _check_eps(eps, "TVNorm")
        self.weight = torch.nn.Parameter(torch.ones(channels, device=device, dtype=dtype))
        with_bias = kind == "layer" if bias is None else bias
        self.bias = torch.nn.Parameter(torch.zeros(channels, device=device, dtype=dtype)) if with_bias else None

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return tv_norm(x, self.weight, self.bias, self.kind, self.eps)

    def extra_repr(self) -> str:
        return "%d, kind=%s, bias=%s" % (self.weight.shape[0], self.kind, self.bias is not None)


class TVResidual(torch.nn.Module):
    """``tv_residual`` with the norm after a block, the scale (init_scale, no scale where it is None) and the norm before the
    next block as parameters.

    ``forward(x, f, gate=None, seed=None, offset=0)`` is y, or (y, h) with a next norm.  Dropout acts in training alone; without a
    seed one is drawn from torch's CPU generator (which a captured graph would repeat: hand it a seed tensor there).  Borders that
    are handed one seed, as those of a stack are, drop the same places unless each has an offset of its own.
    """

    def __init__(self, channels: int, norm: str = "none", next_norm: str = "none", gate_act: str = "none",
                 init_scale: float | None = None, dropout: float = 0.0, eps: float = 1e-6, device=None, dtype=None):
        super().__init__()
        if norm not in _NORMS or next_norm not in _NORMS or gate_act not in _GATE_ACTS:
            raise ValueError("TVResidual: unknown norm %r, next_norm %r or gate_act %r" % (norm, next_norm, gate_act))
        if not 0.0 <= dropout <= 1.0:
            raise ValueError("TVResidual: a probability between 0 and 1 expected, got %r" % (dropout,))
        if not 1 <= channels <= _b.TV_MAX_LENGTH:
            raise ValueError("TVResidual: 1 to %d channels expected" % _b.TV_MAX_LENGTH)
        self.gate_act, self.dropout, self.eps = gate_act, float(dropout), _check_eps(eps, "TVResidual")
        like = dict(eps=eps, device=device, dtype=dtype)
        self.norm = TVNorm(channels, norm, **like) if norm != "none" else None
        self.next = TVNorm(channels, next_norm, **like) if next_norm != "none" else None
        self.scale = None
        if init_scale is not None:
            self.scale = torch.nn.Parameter(torch.full((channels,), float(init_scale), device=device, dtype=dtype))

    def forward(self, x: torch.Tensor, f: torch.Tensor, gate: torch.Tensor | None = None, seed=None, offset: int = 0):
        p = self.dropout if self.training else 0.0
        if p and seed is None:
            seed = int(torch.randint(0, (1 << 63) - 1, ()))
        norm, after = self.norm, self.next
        return tv_residual(x, f, "none" if norm is None else norm.kind, None if norm is None else norm.weight,
                           None if norm is None else norm.bias, gate, self.gate_act if gate is not None else "none", self.scale, p,
                           seed, offset, "none" if after is None else after.kind, None if after is None else after.weight,
                           None if after is None else after.bias, self.eps)

    def extra_repr(self) -> str:
        return "gate_act=%s, scale=%s, dropout=%g" % (self.gate_act, self.scale is not None, self.dropout)
