"""Channel products whose rows are so long that a tile of them spans more than 2^32 bytes.  Whole numbers, so that every
sum is exact and every output has one right value."""
import pytest
import torch

pytestmark = pytest.mark.gpu

LONG, CHUNK = 36_000_000, 1 << 20
BF = torch.bfloat16


def signs(rows, cols, gen):
    """-1, 0 or 1."""
    t = torch.empty(rows, cols, dtype=BF, device="cuda")
    for r in range(0, cols if cols > rows else rows, CHUNK):
        part = t[:, r:r + CHUNK] if cols > rows else t[r:r + CHUNK]
        part.copy_(torch.randint(-1, 2, part.shape, generator=gen, device="cuda", dtype=torch.int8))
    return t


def linear():
    from paper_2204_03643_amd import linear as module
    return module


def test_long_gradients():
    """64 rows of 36 million gradients through ReLU: dx, dW and db of all of them."""
    lin, M, K, N = linear(), 64, 64, LONG
    gen = torch.Generator(device="cuda").manual_seed(1)
    g, w, x = signs(M, N, gen), signs(N, K, gen), signs(M, K, gen)
    words = torch.randint(-(1 << 31), 1 << 31, (M, -(-N // 32)), generator=gen, device="cuda", dtype=torch.int64).to(torch.int32)
    dx, dw, db = lin.tv_linear_backward(g, x, words, w, "relu", bias_grad=True)
    want = torch.zeros(M, K, device="cuda")
    shifts = torch.arange(32, device="cuda", dtype=torch.int32)
    for n in range(0, N, CHUNK):
        e = min(N, n + CHUNK)
        on = ((words[:, n // 32:-(-e // 32)].unsqueeze(-1) >> shifts) & 1).view(M, -1)[:, :e - n]
        dz = g[:, n:e].float() * on
        want += dz @ w[n:e].float()
        assert torch.equal(dw[n:e].float(), dz.t().contiguous() @ x.float()), n
        assert torch.equal(db[n:e].float(), dz.sum(0)), n
    assert torch.equal(dx, want.to(BF))


@pytest.mark.parametrize("held", ("full", "8bit"))
def test_long_inputs(held):
    """64 rows of 36 million inputs: y, dx and dW, from x as it is and from 8-bit codes."""
    lin, M, K, N = linear(), 64, LONG, 64
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, w, g = signs(M, K, gen), signs(N, K, gen), signs(M, N, gen)
    y = lin.tv_linear(x, w)
    from_x = lin.tv_checkpoint8(x) if held == "8bit" else x
    dx, dw, _ = lin.tv_linear_backward(g, from_x, None, w)
    want = torch.zeros(M, N, device="cuda")
    for k in range(0, K, CHUNK):
        a, b = x[:, k:k + CHUNK].float(), w[:, k:k + CHUNK].float()
        want += a @ b.t().contiguous()
        assert torch.equal(dx[:, k:k + CHUNK].float(), g.float() @ b), k
        assert torch.equal(dw[:, k:k + CHUNK].float(), g.float().t().contiguous() @ a), k
    assert torch.equal(y, want.to(BF))


def test_long_outputs():
    """64 rows of 36 million outputs: y with bias, ReLU and residual, and the signs that are held."""
    lin, M, K, N = linear(), 64, 64, LONG
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, w, r = signs(M, K, gen), signs(N, K, gen), signs(M, N, gen)
    b = signs(1, N, gen)[0]
    y, words, _ = lin._forward(x, K, w, K, b, r, "relu", "full")
    shifts = torch.arange(32, device="cuda", dtype=torch.int32)
    for n in range(0, N, CHUNK):
        e = min(N, n + CHUNK)
        z = x.float() @ w[n:e].float().t().contiguous() + b[n:e].float()
        assert torch.equal(y[:, n:e].float(), z.clamp(min=0) + r[:, n:e].float()), n
        on = ((words[:, n // 32:-(-e // 32)].unsqueeze(-1) >> shifts) & 1).view(M, -1)[:, :e - n]
        assert torch.equal(on.bool(), z > 0), n
