"""Forward-mode differentiation of the channel products is refused, not answered without a tangent."""
import pytest
import torch
from torch.autograd import forward_ad

pytestmark = pytest.mark.gpu


def tensors():
    gen = torch.Generator(device="cuda").manual_seed(0)
    return [torch.randn(*s, generator=gen, device="cuda") for s in ((5, 8), (6, 8), (6,), (5, 6))]


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("grad_mode", (True, False))
def test_a_tangent_of_any_input_is_refused(which, grad_mode):
    from paper_2204_03643_amd.linear import tv_linear
    plain = tensors()
    with forward_ad.dual_level(), torch.set_grad_enabled(grad_mode):
        dual = list(plain)
        dual[which] = forward_ad.make_dual(plain[which], torch.ones_like(plain[which]))
        with pytest.raises(NotImplementedError):
            tv_linear(*dual, act="gelu")
        # an open level alone changes nothing
        assert torch.equal(tv_linear(*plain, act="gelu"), tv_linear(*plain, act="gelu"))


def test_tangents_of_gradients_are_refused():
    from paper_2204_03643_amd.linear import tv_linear, tv_linear_backward
    x, w, b, r = tensors()
    g = torch.ones(5, 6, device="cuda")
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(g, torch.ones_like(g))
        y = tv_linear(x.requires_grad_(), w, b, r)
        with pytest.raises(NotImplementedError):
            torch.autograd.grad(y, x, dual)
        with pytest.raises(NotImplementedError):
            tv_linear_backward(dual, x.detach(), None, w)
        with pytest.raises(NotImplementedError):
            tv_linear_backward(g, x.detach(), None, forward_ad.make_dual(w, torch.ones_like(w)))


def test_function_transforms_are_refused():
    from paper_2204_03643_amd.linear import tv_linear
    x, w, b, r = tensors()
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda v: tv_linear(v, w, b, r), (x,), (x,))
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda v: tv_linear(v, w, b))(x)
