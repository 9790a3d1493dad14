"""Gradients of the channel products with their saved tensors kept elsewhere between the passes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("checkpoint", ("full", "8bit"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_saved_on_the_host(dtype, checkpoint):
    """Views of wider tensors come back dense; the gradients keep their bits where the kernels' choice does not go by strides."""
    from paper_2204_03643_amd.linear import tv_linear
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, w, g = (torch.randn(*s, generator=gen, device="cuda").to(dtype) for s in ((130, 320), (72, 256), (130, 72)))
    for act in ("none", "relu", "gelu"):
        grads = []
        for hooks in (torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t), torch.autograd.graph.save_on_cpu()):
            leaves = [x[:, 8:200].detach().requires_grad_(), w[:, 16:208].detach().requires_grad_()]
            with hooks:
                y = tv_linear(*leaves, act=act, checkpoint=checkpoint)
            grads.append(torch.autograd.grad(y, leaves, g))
        for a, b in zip(*grads):
            assert torch.equal(a, b), act
