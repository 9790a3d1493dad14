"""Residual borders, dropout, the TV pass, the channel products and products in 4 bits together, as a network uses them."""
import blockref
import pytest
import quant4ref
import torch

pytestmark = pytest.mark.gpu


def plain(f, x, gate, seed, p, block):
    """The block's steps in torch, f32."""
    from paper_2204_03643_amd.layer import tv_prox_1d
    F = torch.nn.functional
    n = x.shape[-1]
    before = F.layer_norm(x, (n,), f["norm.weight"], f["norm.bias"], 1e-6)
    s = tv_prox_1d(before, F.softplus(f["raw_lambda"]), axis=1)
    h = F.gelu(s @ f["expand.weight"].T + f["expand.bias"]) @ f["reduce.weight"].T + f["reduce.bias"]
    h = h * (h.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * f["residual.norm.weight"]
    c = f["residual.scale"] * torch.sigmoid(gate) * h
    if p:
        keep, factor = blockref.kept(x.shape[0] * x.shape[1], n, p, seed, 0)
        c = torch.where(keep.view(x.shape).to(x.device), c * factor, 0.0)
    return x + c


@pytest.mark.parametrize("p", (0.0, 0.2))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_block_against_the_same_steps_in_torch(dtype, p):
    from paper_2204_03643_amd.linear import TVMixer
    torch.manual_seed(0)
    block = TVMixer(24, 96, checkpoint="full", device="cuda", dtype=dtype, norm="layer", post_norm="rms", init_scale=0.7,
                    dropout=p, gate_act="sigmoid")
    x = torch.randn(3, 50, 24, device="cuda").to(dtype).requires_grad_()
    gate = torch.randn(3, 1, 24, device="cuda").to(dtype).requires_grad_()
    g = torch.randn(3, 50, 24, device="cuda").to(dtype)
    y = block(x, gate, seed=17)
    names = [k for k, _ in block.named_parameters()]
    assert names == ["raw_lambda", "expand.weight", "expand.bias", "reduce.weight", "reduce.bias", "norm.weight", "norm.bias",
                     "residual.scale", "residual.norm.weight"]
    got = torch.autograd.grad(y, [x, gate] + list(block.parameters()), g)
    f = {k: v.detach().float().requires_grad_() for k, v in block.named_parameters()}
    xf, gf = (t.detach().float().requires_grad_() for t in (x, gate))
    yf = plain(f, xf, gf, 17, p, block)
    want = torch.autograd.grad(yf, [xf, gf] + [f[k] for k in names], g.float())
    # bf16: six tensors between are rounded, 2^-8 each at most, and the norms pass on what differs
    off = 0.03 if dtype == torch.bfloat16 else 1e-4
    assert (y.float() - yf).norm() <= off * yf.norm()
    for k, a, b in zip(["x", "gate"] + names, got, want):
        assert a.shape == b.shape and (a.float() - b).norm() <= off * b.norm() + 1e-6, k


def test_a_stack_in_training_and_in_4_bits():
    """Two blocks take a step of training; then they serve in 4 bits, as the same steps with restored weights and activations."""
    from paper_2204_03643_amd.layer import tv_prox_1d
    from paper_2204_03643_amd.linear import TVMixer
    torch.manual_seed(2)
    stack = torch.nn.Sequential(*(TVMixer(64, 256, device="cuda", dtype=torch.bfloat16, norm="rms", init_scale=0.5, dropout=0.1) for _ in range(2)))
    x = torch.randn(2, 40, 64, device="cuda").bfloat16()
    before = [p.detach().clone() for p in stack.parameters()]
    stack(x).float().square().mean().backward()
    torch.optim.SGD(stack.parameters(), lr=0.1).step()
    assert all(p.grad is not None and p.grad.isfinite().all() for p in stack.parameters())
    assert any(not torch.equal(a, b) for a, b in zip(before, stack.parameters()))
    serving = [b.quantized4() for b in stack]
    assert stack[0].training and not serving[0].training

    def held(v):
        rows = v.reshape(-1, v.shape[-1])
        return torch.from_numpy(quant4ref.load(*quant4ref.save(rows.double().cpu().numpy()), v.shape[-1])).to(v.device).view(v.shape)

    def product(v, linear):
        return (held(v) @ held(linear.weight.detach()).T + linear.bias.detach().double())
    y = x
    for block, small in zip(stack.eval(), serving):
        with torch.no_grad():
            got = small(y)
            n = block.norm(y)
            s = tv_prox_1d(n.float(), torch.nn.functional.softplus(block.raw_lambda), axis=1).bfloat16()
            h = torch.nn.functional.gelu(product(s, block.expand)).bfloat16()
            want = y.double() + block.residual.scale.double() * product(h, block.reduce).bfloat16().double()
        # h's rounding may fall on either side and then on either side of a border of 4 bits: about a percent of its norm
        assert (got.double() - want).norm() <= 0.01 * want.norm()
        y = got


@pytest.mark.parametrize("more", ((), ("--norm", "rms", "--dropout", "0.1")))
def test_the_example_runs(more, monkeypatch, capsys):
    import importlib.util
    import os
    import sys
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "denoise_tokens.py")
    spec = importlib.util.spec_from_file_location("denoise_tokens", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", [path, "--steps", "3", "--tokens", "64", "--channels", "16", *more])
    example.main()
    assert "in 4 bits" in capsys.readouterr().out
