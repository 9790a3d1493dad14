"""One seed for a stack of blocks: their offsets tell their masks apart."""
import pytest
import torch

from paper_2204_03643_amd import block
from paper_2204_03643_amd.linear import TVMixer


def test_modules_hand_their_offset_on(monkeypatch):
    seen = []
    monkeypatch.setattr(block, "tv_residual", lambda *a: seen.append(a[9:11]) or a[0])
    x = torch.zeros(2, 3, 8)
    border = block.TVResidual(8, dropout=0.5)
    border(x, x, seed=4)
    border(x, x, None, 4, 7)
    border(x, x, seed=4, offset=1 << 40)
    assert seen == [(4, 0), (4, 7), (4, 1 << 40)]


def test_a_border_in_training_within_a_block_that_is_not(monkeypatch):
    """Dropout goes by the border's own mode, whichever else the border does."""
    from paper_2204_03643_amd import linear

    class Product(torch.nn.Module):
        def forward(self, x, residual=None):
            return x if residual is None else x + residual
    seen = []
    monkeypatch.setattr(linear, "tv_prox_1d", lambda x, lam, axis: x)
    monkeypatch.setattr(block, "tv_residual", lambda *a: seen.append(a[8]) or a[0])
    x = torch.zeros(1, 2, 8)
    for init_scale in (None, 1.0):
        mixer = TVMixer(8, 16, dropout=0.5, init_scale=init_scale)
        mixer.expand = mixer.reduce = Product()
        seen.clear()
        mixer(x)
        mixer.eval()
        mixer.residual.train()
        mixer(x)
        assert seen == [0.5, 0.5]


@pytest.mark.gpu
def test_masks_of_a_stack_with_one_seed_tensor():
    seed = torch.tensor([11], device="cuda")
    stack = [TVMixer(16, 32, device="cuda", dropout=0.5) for _ in range(2)]
    x = torch.randn(2, 60, 16, device="cuda")
    with torch.no_grad():
        for b in stack:
            b.reduce.bias.fill_(100.0)               # so that what is kept differs from x

        def dropped(b, offset):
            return b(x, None, seed, offset) == x
        a, other = dropped(stack[0], 0), dropped(stack[1], 1)
        assert 0.4 < a.float().mean().item() < 0.6 and 0.4 < other.float().mean().item() < 0.6
        # independent halves: 1920 places, five standard deviations
        assert abs((a == other).float().mean().item() - 0.5) <= 5 * 0.5 / 1920 ** 0.5
        assert torch.equal(dropped(stack[1], 0), a) and torch.equal(dropped(stack[0], 1), other)
        assert torch.equal(block.tv_dropout(torch.ones_like(x), 0.5, 11, 1) == 0, other)
        assert torch.equal(stack[0](x, seed=seed), stack[0](x, None, 11, 0))
    # the backward pass drops what the forward pass did
    border = block.TVResidual(16, dropout=0.5, device="cuda")
    f = torch.randn(2, 60, 16, device="cuda", requires_grad=True)
    g = torch.autograd.grad(border(x, f, seed=seed, offset=1).sum(), f)[0]
    assert torch.equal(g == 0, other)
