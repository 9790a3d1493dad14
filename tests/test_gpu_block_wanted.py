"""Backward calls of residual borders where some of the gradients are wanted, against 64 bits."""
import blockref
import pytest
import torch
from test_gpu_block import NAMES, check, made, wide

pytestmark = pytest.mark.gpu

ALL = ("x", "f") + NAMES
# what is frozen; the rest is trained
FROZEN = [("bias",), ("weight",), ("gate",), ("scale",), ("x",), ("f",), ("next_weight",), ("next_bias",), ("x", "f"), ("weight", "bias"),
          ("weight", "scale"), ("bias", "scale"), ("weight", "bias", "scale"), ("next_weight", "next_bias"), ("x", "f", "gate", "next_weight", "next_bias"),
          ("x", "bias", "gate"), tuple(k for k in ALL if k != "x"), tuple(k for k in ALL if k != "f")] + [
          tuple(k for k in ALL if k != name) for name in NAMES]


def gradients(t, frozen, shape, gate_shape, **how):
    """{name: tensor} of tv_residual's outputs and of the gradients that are wanted."""
    from paper_2204_03643_amd.block import tv_residual
    c = {k: None if v is None else v.cuda() for k, v in t.items()}
    for k in ("x", "f", "dy", "dh"):
        c[k] = None if c[k] is None else c[k].reshape(shape)
    if c["gate"] is not None:
        c["gate"] = c["gate"].reshape(gate_shape)
    leaves = [k for k in ALL if c[k] is not None and k not in frozen]
    for k in leaves:
        c[k].requires_grad_()
    out = tv_residual(c["x"], c["f"], **{k: c[k] for k in NAMES}, **how)
    out = out if isinstance(out, tuple) else (out,)
    torch.autograd.backward(out, [c["d" + k] for k in ("y", "h")[:len(out)]])
    got = dict(zip(("y", "h"), (a.detach() for a in out)))
    got.update(("d" + k, c[k].grad) for k in leaves)
    assert all(c[k].grad is None for k in ALL if c[k] is not None and k not in leaves)
    return got


@pytest.mark.parametrize("frozen", FROZEN, ids="-".join)
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("m,n,gate", [(30, 72, 5), (30, 1001, 1), (30, 4104, 6), (33, 8191, 3), (20, 8200, 4), (12, 4104, 12)])
def test_some_gradients_are_wanted(m, n, gate, dtype, frozen):
    """Up to 4096 channels the sums over rows lie in registers, with more in LDS or in a pass of their own; which, and where each
    sum is put, goes by which gradients are wanted."""
    how = dict(norm="layer", next_norm="layer", gate_act="sigmoid")
    t = made(m, n, dtype, m + n, "layer", "layer", True, gate, True)
    got = gradients(t, frozen, (gate, m // gate, n), (gate, 1, n), dropout=0.1, seed=3, **how)
    check(t, dtype, got, p=0.1, seed=3, **how)


@pytest.mark.parametrize("frozen", [(), ("f",), ("x",), ("next_weight",), ("x", "f")], ids="-".join)
@pytest.mark.parametrize("n", (200, 5000, 9000))
def test_some_gradients_are_wanted_without_a_gate(n, frozen):
    how = dict(norm="none", next_norm="rms")
    t = made(7, n, torch.float32, n, "none", "rms", False, 0, False)
    got = gradients(t, frozen, (7, n), None, dropout=0.3, seed=8, **how)
    check(t, torch.float32, got, p=0.3, seed=8, **how)


@pytest.mark.parametrize("frozen", [("x",), ("next_weight",), ("next_bias",), ("x", "next_bias"), ("x", "next_weight"), ("next_weight", "next_bias")],
                         ids="-".join)
@pytest.mark.parametrize("n", (72, 2047, 8192, 8200))
def test_some_gradients_of_a_norm_are_wanted(n, frozen):
    from paper_2204_03643_amd.block import tv_norm
    t = made(9, n, torch.bfloat16, n, "none", "layer", True, 0, False)
    c = {k: t[k].cuda().requires_grad_(k not in frozen) for k in ("x", "next_weight", "next_bias")}
    tv_norm(c["x"], c["next_weight"], c["next_bias"], kind="layer").backward(t["dh"].cuda())
    ref = wide(t)
    want = blockref.border(torch.bfloat16, ref["x"], next_norm="layer", next_weight=ref["next_weight"], next_bias=ref["next_bias"], dh=ref["dh"])
    for k, v in c.items():
        assert (v.grad is None) == (k in frozen)
        if v.grad is not None:
            blockref.within(v.grad, want["d" + k], "d" + k)
