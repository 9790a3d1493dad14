"""Dropout of a single number."""
import blockref
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_number_that_stands_for_the_negative_of_its_memory():
    from paper_2204_03643_amd.block import tv_dropout
    v = torch.tensor(1 + 2j, device="cuda").conj().imag
    assert v.is_neg() and v.dim() == 0
    seed = next(s for s in range(100) if bool(blockref.kept(1, 1, 0.5, s, 0)[0]))
    assert tv_dropout(v, 0.5, seed).item() == -4.0
    leaf = torch.tensor(1.0, device="cuda", requires_grad=True)
    assert torch.autograd.grad(tv_dropout(leaf, 0.5, seed), leaf, v)[0].item() == -4.0
