"""Dropout from the counter-based generator, against the generator's definition."""
import blockref
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("rows,n,p,seed,offset", [(1, 1, 0.5, 1, 0), (3, 7, 0.25, 0, 0), (5, 8, 0.9, -1, 5), (2, 9, 0.1, 1 << 63, 1 << 32),
                                                  (257, 101, 0.25, 123456789012345, (1 << 64) - 1), (4, 2049, 1.0 / 65536, 3, 2),
                                                  (300, 64, 0.99999, 5, 1), (9, 16500, 0.5, 77, 0), (1, 5000, 1.0, 2, 2), (70, 264, 0.3, 8, 8)])
def test_what_is_dropped(rows, n, p, seed, offset, dtype):
    from paper_2204_03643_amd.block import tv_dropout
    gen = torch.Generator().manual_seed(rows + n)
    x, g = (torch.randn(rows, n, generator=gen).to(dtype) for _ in range(2))
    leaf = x.cuda().requires_grad_()
    y = tv_dropout(leaf, p, seed, offset)
    dx = torch.autograd.grad(y, leaf, g.cuda())[0]
    keep, factor = blockref.kept(rows, n, p, seed, offset)
    for got, v in ((y, x), (dx, g)):
        want = torch.where(keep, v.double() * factor, 0.0)
        # the factor's rounding, the product's, and the output's
        blockref.within(got, (want, want.abs() * (3 * blockref.U32 + blockref.unit(dtype))), "dropout")
        assert bool((got.detach().cpu()[~keep] == 0).all())
    with torch.no_grad():
        assert torch.equal(tv_dropout(leaf, p, seed, offset), y)


def test_the_generator_gives_the_numbers_of_its_paper():
    """The known answers of Philox 4x32-10, of the reference here that the kernels are held to."""
    def words(seed, counter):
        return [int(w) for w in blockref.philox(seed, counter)]
    assert words(0, [0, 0, 0, 0]) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    full = (1 << 32) - 1
    assert words((1 << 64) - 1, [full] * 4) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert words(0x299F31D0A4093822, [0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_how_much_is_dropped():
    from paper_2204_03643_amd.block import tv_dropout
    x = torch.ones(4096, 1024, device="cuda")
    for p in (0.1, 0.5):
        gone = tv_dropout(x, p, 4) == 0
        # 4M draws: five standard deviations of the whole, and of a row's share
        assert abs(gone.float().mean().item() - p) <= 5 * (p * (1 - p) / gone.numel()) ** 0.5 + 2.0 ** -17
        # (the largest of 4096 rows; six deviations)
        assert (gone.float().mean(1) - p).abs().max().item() <= 6 * (p * (1 - p) / 1024) ** 0.5
    a, b, c = (tv_dropout(x, 0.5, s, o) for s, o in ((4, 0), (5, 0), (4, 1)))
    for other in (b, c):
        assert abs(((a == 0) == (other == 0)).float().mean().item() - 0.5) < 0.01


def test_what_is_dropped_is_zero_whatever_it_was():
    from paper_2204_03643_amd.block import tv_dropout
    x = torch.full((3, 1000), float("nan"), device="cuda")
    x[1], x[2] = float("inf"), float("-inf")
    keep, _ = blockref.kept(3, 1000, 0.5, 6, 0)
    y = tv_dropout(x, 0.5, 6).cpu()
    assert bool((y[~keep] == 0).all()) and not bool(y[keep].isfinite().any())


def test_seeds_on_the_device():
    from paper_2204_03643_amd.block import tv_dropout
    x = torch.randn(5, 100, device="cuda")
    for s in (0, 3, -7, (1 << 62) + 5):
        at = torch.tensor([s], device="cuda")
        assert torch.equal(tv_dropout(x, 0.4, at, 9), tv_dropout(x, 0.4, s, 9))
    leaf = x.clone().requires_grad_()
    at = torch.tensor(3, device="cuda")
    y = tv_dropout(leaf, 0.4, at)
    at.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    with pytest.raises(TypeError):
        tv_dropout(x, 0.4, torch.tensor([1.0], device="cuda"))
    with pytest.raises(TypeError):
        tv_dropout(x, 0.4, torch.tensor([1]))


def test_rows_past_32_bits():
    """Rows 2^30 values apart, so that the last starts 2^32 values from the first."""
    from paper_2204_03643_amd.block import tv_dropout, tv_norm
    base = torch.empty((1 << 32) + 64, dtype=torch.bfloat16, device="cuda")
    x = base.as_strided((5, 40), (1 << 30, 1))
    x.copy_(torch.randn(5, 40, device="cuda"))
    dense = x.contiguous()
    assert torch.equal(tv_dropout(x, 0.5, 1), tv_dropout(dense, 0.5, 1))
    assert torch.equal(tv_norm(x), tv_norm(dense))


def test_more_rows_than_a_launch_has_workgroups():
    from paper_2204_03643_amd.block import tv_dropout
    rows, n = 300001, 12
    y = tv_dropout(torch.ones(rows, n, device="cuda"), 0.4, 9)
    some = [0, 1, 262143, 262144, 300000]
    keep, _ = blockref.kept(some, n, 0.4, 9, 0)
    assert torch.equal(y[some].cpu() != 0, keep)


def test_shapes():
    from paper_2204_03643_amd.block import tv_dropout
    x = torch.randn(6, 50, device="cuda")
    y = tv_dropout(x, 0.5, 1)
    assert torch.equal(tv_dropout(x.view(2, 3, 50), 0.5, 1).view(6, 50), y)
    assert torch.equal(tv_dropout(x[0], 0.5, 1), y[0])
    wide = torch.randn(6, 121, device="cuda")
    assert torch.equal(tv_dropout(wide[:, 7:57], 0.5, 1), tv_dropout(wide[:, 7:57].contiguous(), 0.5, 1))
    assert tv_dropout(torch.tensor(2.0, device="cuda"), 0.5, 1).shape == ()
    assert torch.equal(tv_dropout(x, 0.0, None), x) and torch.equal(tv_dropout(x, 2.0 ** -18, 1), x)
