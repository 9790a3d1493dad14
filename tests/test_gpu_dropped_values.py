"""Values that dropout takes out, which have no part in outputs or gradients, whatever they are."""
import blockref
import pytest
import torch
from test_gpu_block import NAMES, made

pytestmark = pytest.mark.gpu

ODD = (float("nan"), float("inf"), float("-inf"))


def step(t, shape, **how):
    """Outputs and gradients of a border."""
    from paper_2204_03643_amd.block import tv_residual
    c = {k: v.cuda().reshape(shape) if v.dim() == 2 else v.cuda() for k, v in t.items() if v is not None}
    leaves = [k for k in ("x", "f") + NAMES if k in c]
    for k in leaves:
        c[k].requires_grad_()
    out = tv_residual(c["x"], c["f"], **{k: c.get(k) for k in NAMES}, dropout=0.5, seed=5, offset=2, **how)
    out = dict(zip(("y", "h"), out if isinstance(out, tuple) else (out,)))
    grads = torch.autograd.grad(list(out.values()), [c[k] for k in leaves], [c["d" + k] for k in out])
    return {**{k: v.detach() for k, v in out.items()}, **{"d" + k: g for k, g in zip(leaves, grads)}}


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("m,n", [(12, 200), (12, 201), (3, 2048), (9, 5000), (4, 9000)])
@pytest.mark.parametrize("norm,next_norm,act,scale", [("none", "none", "none", False), ("none", "none", None, True), ("none", "rms", "silu", True), ("layer", "layer", "sigmoid", True),
                                                      ("rms", "none", "none", True), ("rms", "layer", "silu", True)])
def test_what_was_dropped_has_no_part_in_gradients(m, n, norm, next_norm, act, scale, dtype):
    t = made(m, n, dtype, m + n, norm, next_norm, norm == "layer", m if act is not None else 0, scale)
    keep, _ = blockref.kept(m, n, 0.5, 5, 2)
    how = dict(norm=norm, next_norm=next_norm, gate_act=act or "none")
    spoiled = dict(t)
    # f where it isn't normed (a norm takes in its whole row), and a gate of its own for each row
    names = (["f"] if norm == "none" else []) + (["gate"] if act is not None else []) + (["dy"] if next_norm == "none" else [])
    gone = (~keep).nonzero()
    for j, k in enumerate(names):
        spoiled[k] = t[k].clone()
        some = gone[j::7]
        spoiled[k][some[:, 0], some[:, 1]] = torch.tensor(ODD, dtype=dtype)[torch.arange(len(some)) % 3]
    assert names and not all(spoiled[k].isfinite().all() for k in names)
    want, got = step(t, (m, n), **how), step(spoiled, (m, n), **how)
    for k, v in got.items():
        if k == "dx" and next_norm == "none":                        # (is dy)
            continue
        assert torch.equal(v, want[k]), k
