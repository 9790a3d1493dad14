"""The backward pass of the channel products and hooks on saved tensors (no GPU needed: the kernels are replaced)."""
import pytest
import torch

from paper_2204_03643_amd import linear as lin


def rows_in_memory(t, ld):
    """What a kernel finds that is told of dense rows ld apart."""
    count = t.numel() // t.shape[-1]
    raw = torch.empty(0, dtype=t.dtype).set_(t.untyped_storage())
    assert t.storage_offset() + (count - 1) * ld + t.shape[-1] <= raw.numel(), "rows end past the memory"
    return torch.as_strided(raw, (count, t.shape[-1]), (ld, 1), t.storage_offset())


@pytest.fixture
def seen(monkeypatch):
    """The operands that the backward call is given, as its kernels would read them."""
    found = {}

    def forward(x, ldx, weight, ldw, bias, residual, act, hold):
        z = rows_in_memory(x, ldx) @ rows_in_memory(weight, ldw).t()
        return z.clone(), z, None

    def backward(g, x, x_exps, ldx, data, exps, weight, ldw, act, want):
        found.update(x=rows_in_memory(x, ldx).clone(), w=rows_in_memory(weight, ldw).clone(), z=rows_in_memory(data, data.shape[-1]).clone())
        return torch.zeros(g.shape[0], weight.shape[1]), torch.zeros(weight.shape), None
    monkeypatch.setattr(lin, "_forward", forward)
    monkeypatch.setattr(lin, "_backward", backward)
    monkeypatch.setattr(lin, "_check_tensor", lambda t, what, like=None: t)
    return found


HOOKS = {"none": (lambda t: t, lambda t: t),
         "dense copies": (lambda t: t.contiguous().clone(), lambda t: t),
         "rows further apart": (lambda t: torch.nn.functional.pad(t, (0, 5))[:, :t.shape[1]], lambda t: t),
         "columns first": (lambda t: t.t().contiguous(), lambda t: t.t())}


@pytest.mark.parametrize("hook", HOOKS)
def test_strides_are_those_of_the_tensors_that_come_back(seen, hook):
    """torch.autograd.graph.save_on_cpu, for one, brings back dense tensors for views of wider ones."""
    x = torch.randn(6, 40)[:, 3:11].requires_grad_()
    w = torch.randn(5, 30)[:, :8].requires_grad_()
    with torch.autograd.graph.saved_tensors_hooks(*HOOKS[hook]):
        y = lin._Linear.apply(x, w, None, None, "gelu", "full")
    y.backward(torch.ones(6, 5))
    assert torch.equal(seen["x"], x.detach()) and torch.equal(seen["w"], w.detach())
    assert torch.equal(seen["z"], y.detach())


@pytest.mark.parametrize("change", (lambda t: t.double(), lambda t: t[:-1], lambda t: t.flatten(), lambda t: t.to("meta")))
def test_other_tensors_are_refused(seen, change):
    x, w = torch.randn(6, 8, requires_grad=True), torch.randn(5, 8, requires_grad=True)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
        y = lin._Linear.apply(x, w, None, None, "gelu", "full")
    with pytest.raises(RuntimeError, match="saved tensors"):
        y.backward(torch.ones(6, 5))
