"""f32 channel products to the last bit where sums have one term, and in the 2-norm where they have many: a tolerance for sums of
many terms alone would not miss a partial product of the bf16 parts."""
import pytest
import torch

import splitref as ref

pytestmark = pytest.mark.gpu

# every size of f32 tiles, contractions in one piece and in several, tiles that end early, few rows
SHAPES = [(4096, 192, 4096), (4096, 4096, 4096), (2048, 2048, 2048), (4096, 1024, 1024), (300, 64, 260), (264, 2048, 200),
          (513, 1027, 258), (1100, 328, 1161), (7, 1001, 777)]


def linear():
    from paper_2204_03643_amd import linear as module
    return module


def cuda(*tensors):
    return [t.cuda().contiguous() for t in tensors]


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_one_term(M, K, N):
    lin = linear()
    a, b, d = cuda(*ref.one_term(M, N, K, M + K))                    # y = a b^T
    assert torch.equal(lin.tv_linear(a, b), d)
    a, b, d = cuda(*ref.one_term(N, M, K, M + K + 1))                # the other way round: x has one value a row
    assert torch.equal(lin.tv_linear(b, a), d.t())
    x, w = torch.zeros(M, K, device="cuda"), torch.zeros(N, K, device="cuda")
    a, b, d = cuda(*ref.one_term(M, K, N, M + K + 2))                # dx = g W
    assert torch.equal(lin.tv_linear_backward(a, x, None, b.t().contiguous())[0], d)
    a, b, d = cuda(*ref.one_term(K, M, N, M + K + 3))
    assert torch.equal(lin.tv_linear_backward(b, x, None, a.t().contiguous())[0], d.t())
    a, b, d = cuda(*ref.one_term(N, K, M, M + K + 4))                # dW = g^T x
    assert torch.equal(lin.tv_linear_backward(a.t().contiguous(), b.t().contiguous(), None, w)[1], d)
    a, b, d = cuda(*ref.one_term(K, N, M, M + K + 5))
    assert torch.equal(lin.tv_linear_backward(b.t().contiguous(), a.t().contiguous(), None, w)[1], d.t())
    a, b, d = cuda(*ref.one_term(N, K, M, M + K + 6, ones=True))     # from codes, which hold +-1 exactly
    held = lin.tv_checkpoint8(b.t().contiguous())
    assert torch.equal(held.restore(), b.t())
    assert torch.equal(lin.tv_linear_backward(a.t().contiguous(), held, None, w)[1], d)


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_many_terms_in_the_2_norm(M, K, N):
    """n terms of random signs: each addition rounds by at most half a unit of a partial sum, of which the i-th is sqrt(i)
    terms large: together at most sqrt(n) half units of the result, and two for the parts that are left out and the rounding."""
    lin = linear()
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    x, w, g = (torch.randn(*s, generator=gen, device="cuda") for s in ((M, K), (N, K), (M, N)))
    held = lin.tv_checkpoint8(x)

    def near(got, want, terms):
        assert ref.relative_error(got, want) <= (2 + terms ** 0.5) * 2.0 ** -24
    near(lin.tv_linear(x, w), x.double() @ w.double().t().contiguous(), K)
    dx, dw, _ = lin.tv_linear_backward(g, x, None, w)
    gt = g.double().t().contiguous()
    near(dx, g.double() @ w.double(), N)
    near(dw, gt @ x.double(), M)
    near(lin.tv_linear_backward(g, held, None, w)[1], gt @ held.restore().double(), M)


@pytest.mark.parametrize("M,K,N", [(300, 64, 260), (2048, 2048, 2048), (4096, 192, 4096), (264, 2048, 200)])
def test_values_whose_parts_leave_bf16_range(M, K, N):
    """Below 2^-110 the last bits of an f32 value lie below bf16's least number, 2^-133: a value is then taken to half of
    that, 2^-134, and the products are off by that much of the other operand on top of the usual bound."""
    lin = linear()
    gen = torch.Generator(device="cuda").manual_seed(K)
    for e in (-105, -115, -125):
        x = torch.randn(M, K, generator=gen, device="cuda") * 2.0 ** e
        w = torch.randn(N, K, generator=gen, device="cuda") * 2.0 ** 20
        x64, w64 = x.double(), w.double()
        size, other = x64.abs() @ w64.t().abs().contiguous(), w64.abs().sum(1)
        off = (K + 8) * 2.0 ** -24 * size + 2.0 ** -134 * other + 2.0 ** -149
        assert ((lin.tv_linear(x, w).double() - x64 @ w64.t().contiguous()).abs() <= off).all(), e
