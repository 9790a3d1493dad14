"""What the exact tests of f32 products can see, on the CPU: every partial product that is left out."""
import itertools

import pytest
import torch

import splitref as ref

SIX = [(i, j) for i, j in itertools.product(range(3), range(3)) if i + j <= 2]


def test_six_partial_products_are_enough():
    for a, b, d in (ref.one_term(60, 90, 200, 1), ref.one_term(60, 90, 200, 2, ones=True)):
        assert torch.equal(ref.from_parts(a, b), d)
        assert torch.equal(ref.from_parts(b, a), d.t())


@pytest.mark.parametrize("missing", SIX)
def test_each_of_the_six_is_needed(missing):
    a, b, d = ref.one_term(60, 90, 200, 3)
    assert not torch.equal(ref.from_parts(a, b, [missing]), d)
    assert not torch.equal(ref.from_parts(b, a, [missing]), d.t())


@pytest.mark.parametrize("missing", [(0, 0), (1, 0), (2, 0)])
def test_each_of_the_three_against_codes_is_needed(missing):
    a, b, d = ref.one_term(60, 90, 200, 4, ones=True)
    assert not torch.equal(ref.from_parts(a, b, [missing]), d)
    assert torch.equal(ref.from_parts(a, b, [p for p in SIX if p[1]]), d)        # B is exact in its first part


@pytest.mark.parametrize("missing", SIX)
def test_the_norm_sees_it_over_short_contractions(missing):
    gen = torch.Generator().manual_seed(5)
    a, b = torch.randn(200, 16, generator=gen), torch.randn(200, 16, generator=gen)
    want = a.double() @ b.double().t()
    limit = (2 + 16 ** 0.5) * 2.0 ** -24
    assert ref.relative_error(ref.from_parts(a, b), want) <= limit
    assert ref.relative_error(ref.from_parts(a, b, [missing]), want) > limit
