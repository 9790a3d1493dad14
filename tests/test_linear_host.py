"""Refusals of the channel products and the 8-bit checkpoints, before any device is touched (no GPU needed)."""
import pytest
import torch

import paper_2204_03643_amd as tv

FAKE = 0x1000
OK, NULL, SHAPE, STRIDE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 5, 6
NOTHING = tv.tv_held(None, None, tv.TV_HELD_NONE)


def desc(m=4, k=32, n=16, ldx=None, ldw=None, ldr=None, ldy=None, dtype=tv.TV_F32, act=tv.TV_ACT_NONE):
    return tv.tv_linear_desc(m, k, n, k if ldx is None else ldx, k if ldw is None else ldw, n if ldr is None else ldr,
                             n if ldy is None else ldy, dtype, act)


def fwd(d, x=FAKE, w=FAKE, bias=None, res=None, y=FAKE, held=NOTHING, ws=None, nbytes=0):
    return tv.lib().tv_linear_fwd(x, w, bias, res, y, held, d, ws, nbytes, None)


def bwd(d, g=FAKE, x=FAKE, exps=None, held=NOTHING, w=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, nbytes=1 << 40):
    return tv.lib().tv_linear_bwd(g, x, exps, held, w, dx, dw, db, d, ws, nbytes, None)


BAD_DESCS = [(desc(m=-1), SHAPE), (desc(k=0), SHAPE), (desc(n=0), SHAPE), (desc(m=1 << 31), SHAPE), (desc(k=1 << 31), SHAPE),
             (desc(n=1 << 31), SHAPE), (desc(m=(1 << 31) - 1, n=(1 << 31) - 1000), SHAPE), (desc(dtype=2), UNSUPPORTED),
             (desc(dtype=-1), UNSUPPORTED), (desc(act=4), UNSUPPORTED), (desc(act=-1), UNSUPPORTED), (desc(ldx=31), STRIDE),
             (desc(ldw=31), STRIDE), (desc(ldy=15), STRIDE), (desc(ldx=1 << 31), STRIDE), (desc(ldw=-32), STRIDE)]


@pytest.mark.parametrize("d,status", BAD_DESCS)
def test_bad_descriptors(d, status):
    assert fwd(d) == status and bwd(d) == status
    assert tv.tv_linear_fwd_workspace_bytes(d) == 0 and tv.tv_linear_bwd_workspace_bytes(d, False) == 0


def test_forward_refusals():
    assert fwd(desc(), x=None) == NULL and fwd(desc(), w=None) == NULL and fwd(desc(), y=None) == NULL
    assert fwd(desc(ldr=15), res=FAKE) == STRIDE
    for name in ("x", "w", "bias", "res", "y"):
        assert fwd(desc(), **{name: FAKE + 2}) == STRIDE
        assert fwd(desc(dtype=tv.TV_BF16), **{name: FAKE + 1}) == STRIDE
    assert fwd(desc(m=0), x=None, w=None, y=None) == OK                      # nothing to do
    assert fwd(desc(m=0, ldx=3), x=None, w=None, y=None) == STRIDE


@pytest.mark.parametrize("act,kind,fine", [(a, k, {0: (0,), 1: (0, 2), 2: (0, 1, 3), 3: (0, 1, 3)}[a].count(k) > 0)
                                           for a in range(4) for k in range(5)])
def test_held_kinds(act, kind, fine):
    """m = 0, so that what is accepted returns without a launch."""
    d = desc(m=0, act=act)
    assert fwd(d, held=tv.tv_held(FAKE, FAKE, kind)) == (OK if fine else UNSUPPORTED)
    d = desc(act=act)
    if fine and kind:
        assert fwd(d, held=tv.tv_held(None, FAKE, kind)) == NULL
        assert bwd(d, held=tv.tv_held(None, FAKE, kind)) == NULL
        if kind == tv.TV_HELD_8BIT:
            assert fwd(d, held=tv.tv_held(FAKE, None, kind)) == NULL
        else:
            assert fwd(d, held=tv.tv_held(FAKE + 2, None, kind)) == STRIDE
    if act and not kind:
        assert bwd(d) == UNSUPPORTED                                         # the backward call needs what the forward held
    if not fine:
        assert bwd(d, held=tv.tv_held(FAKE, FAKE, kind)) == UNSUPPORTED


def test_backward_refusals():
    assert bwd(desc(), g=None) == NULL and bwd(desc(), w=None) == NULL and bwd(desc(), x=None) == NULL
    for name in ("g", "x", "w", "dx", "dw", "db"):
        assert bwd(desc(), **{name: FAKE + 2}) == STRIDE
    need = tv.tv_linear_bwd_workspace_bytes(desc(), False)
    assert need > 0
    assert bwd(desc(), ws=None) == WORKSPACE and bwd(desc(), nbytes=need - 1) == WORKSPACE and bwd(desc(), ws=FAKE + 8) == WORKSPACE
    assert tv.tv_linear_bwd_workspace_bytes(desc(), True) >= need


def test_forward_workspace():
    d = desc(m=64, k=8192, n=256)                                            # few outputs, a long contraction
    need = tv.tv_linear_fwd_workspace_bytes(d)
    assert need > 0
    assert fwd(d, ws=None, nbytes=need) == WORKSPACE and fwd(d, ws=FAKE, nbytes=need - 1) == WORKSPACE
    assert fwd(d, ws=FAKE + 4, nbytes=need) == WORKSPACE


def test_checkpoint_refusals():
    L = tv.lib()
    for call in (lambda a, b, c, rows, n, ld, t: L.tv_ckpt8_save(a, b, c, rows, n, ld, t, None),
                 lambda a, b, c, rows, n, ld, t: L.tv_ckpt8_load(b, c, a, rows, n, ld, t, None)):
        assert call(None, FAKE, FAKE, 2, 40, 40, 0) == NULL and call(FAKE, None, FAKE, 2, 40, 40, 0) == NULL
        assert call(FAKE, FAKE, None, 2, 40, 40, 0) == NULL
        assert call(FAKE, FAKE, FAKE, -1, 40, 40, 0) == SHAPE and call(FAKE, FAKE, FAKE, 2, 0, 40, 0) == SHAPE
        assert call(FAKE, FAKE, FAKE, 1 << 30, 1 << 30, 1 << 30, 0) == SHAPE
        assert call(FAKE, FAKE, FAKE, 2, 40, 39, 0) == STRIDE and call(FAKE + 2, FAKE, FAKE, 2, 40, 40, 0) == STRIDE
        assert call(FAKE, FAKE, FAKE, 2, 40, 40, 7) == UNSUPPORTED
        assert call(None, None, None, 0, 40, 40, 0) == OK


def test_python_refusals():
    from paper_2204_03643_amd import linear as lin
    x, w = torch.zeros(2, 8), torch.zeros(4, 8)
    with pytest.raises(RuntimeError, match="GPU only"):                      # no CPU fallback
        lin.tv_linear(x, w)
    with pytest.raises(RuntimeError, match="GPU only"):
        lin.tv_checkpoint8(x)
    with pytest.raises(RuntimeError, match="GPU only"):
        lin.Checkpoint8(torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8), torch.float32)
    with pytest.raises(TypeError):
        lin.Checkpoint8(x, torch.zeros(2, 1, dtype=torch.uint8), torch.float32)
    with pytest.raises(ValueError):
        lin.Checkpoint8(torch.zeros(2, 33, dtype=torch.int8), torch.zeros(2, 1, dtype=torch.uint8), torch.float32)
    for bad in (dict(act="tanh"), dict(checkpoint="4bit")):
        with pytest.raises(ValueError):
            lin.TVLinear(8, 4, **bad)
    with pytest.raises(ValueError):
        lin.TVLinear(0, 4)
    with pytest.raises(ValueError):
        lin.TVMixer(8, 16, init_lambda=0.0)
    with pytest.raises(ValueError):
        lin.TVMixer(8, 16)(torch.zeros(2, 3, 7))
    block = lin.TVMixer(8, 16, dtype=torch.bfloat16)
    assert block.raw_lambda.dtype == torch.float32 and block.expand.weight.dtype == torch.bfloat16


@pytest.mark.gpu
def test_python_refusals_of_gpu_tensors():
    from paper_2204_03643_amd import linear as lin
    like = dict(device="cuda")
    x, w = torch.zeros(2, 8, **like), torch.zeros(4, 8, **like)
    with pytest.raises(TypeError):
        lin.tv_linear(x.half(), w.half())
    with pytest.raises(TypeError):
        lin.tv_linear(x, w.bfloat16())
    for bad in (dict(weight=torch.zeros(4, 9, **like)), dict(weight=w[0]), dict(bias=torch.zeros(5, **like)),
                dict(residual=torch.zeros(2, 5, **like)), dict(residual=torch.zeros(4, **like)), dict(act="tanh"),
                dict(checkpoint="none")):
        with pytest.raises(ValueError):
            lin.tv_linear(**{"x": x, "weight": w, **bad})
    g = torch.zeros(2, 4, **like)
    for bad in (dict(z=g), dict(act="relu"), dict(act="relu", z=g), dict(act="gelu"), dict(act="gelu", z=g[:, :3]),
                dict(g=g[:1]), dict(act="silu", z=lin.tv_checkpoint8(torch.zeros(2, 5, **like)))):
        with pytest.raises(ValueError):
            lin.tv_linear_backward(**{"g": g, "x": x, "z": None, "weight": w, **bad})
