"""Channel products at sizes that take each of the kernels and ways to split, next to the lines between them, and past
32-bit offsets.  Sampled outputs against 64 bits where all of them would take long."""
import numpy as np
import pytest
import torch

import linref as ref

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# outputs of one workgroup's tile and of several rounds of them, sizes that are multiples of the tiles or one off, short
# and long contractions (one or many splits), and rows that do not start on 16-byte boundaries
SHAPES = [(4096, 192, 4096), (2048, 136, 2048), (4104, 72, 2056), (2049, 96, 2047), (1100, 328, 1160), (257, 4096, 257),
          (96, 8192, 136), (4095, 513, 1025), (40, 640, 1300), (32, 512, 96), (33, 512, 96), (64, 8200, 72), (65, 8200, 72), (8192, 64, 64),
          (130, 63, 4097), (1024, 1000, 1024), (1000, 2500, 64), (4096, 4096, 200), (264, 4096, 4096),
          (32, 1001, 777), (64, 500, 4133), (7, 4096, 5000), (60, 256, 40)]


def linear():
    from paper_2204_03643_amd import linear as module
    return module


def inputs(M, K, N, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    def draw(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)
    return draw(M, K), draw(N, K, scale=K ** -0.5), draw(N), draw(M, N), draw(M, N)


def sample(n, most=48):
    """The first, the last and some indices between, those at tile borders among them."""
    at = {0, n - 1, n // 2, n // 3}
    for b in (32, 64, 128, 256):
        at |= {b - 1, b, n // b * b - 1, n // b * b}
    at |= set(range(7, n, max(1, n // 24)))
    return torch.tensor(sorted(i for i in at if 0 <= i < n)[:most])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_every_kernel(M, K, N, dtype):
    lin, t = linear(), DTYPES[dtype]
    x, w, b, r, g = inputs(M, K, N, t, M + 3 * K + 7 * N)
    x64, w64, b64 = x.double().cpu(), w.double().cpu(), b.double().cpu()
    rows, cols, ks = sample(M), sample(N), sample(K)
    for act, hold in (("gelu", "8bit"), ("relu", "full"), ("none", "full"), ("silu", "full")):
        y, data, exps = lin._forward(x, K, w, K, b, r, act, hold)
        plain = lin._forward(x, K, w, K, b, r, act, None)[0]
        assert torch.equal(y, plain)
        z64, y64, z_off, off = ref.forward(x64[rows], w64, b64, r.double().cpu()[rows], act, t)
        ref.within(y[rows.cuda()], y64, off, ("y", act))
        if act == "none":
            continue
        dx, dw, db = lin._backward(g, x, None, K, data, exps, w, K, act, (True, True, True))
        # the slopes of z as it is held
        if act == "relu":
            words = data.cpu().numpy().view(np.uint32)
            held = torch.from_numpy(((words[:, :, None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(M, -1)[:, :N].astype(np.float64)) * 2 - 1
            sure = z64.abs() > z_off
            assert ((held[rows] > 0) == (z64 > 0))[sure].all()
        elif hold == "8bit":
            held = torch.from_numpy(ref.restored(data.cpu().numpy(), exps.cpu().numpy()))
        else:
            held = data.double().cpu()
            ref.within(data[rows.cuda()], z64, z_off + ref.unit(t) * (z64.abs() + z_off), ("z", act))
        g64 = g.double().cpu()
        (want, _, _), (o, _, _) = ref.backward(g64[rows], x64[rows], held[rows], w64, act, t)
        ref.within(dx[rows.cuda()], want, o, ("dx", act))
        (_, want, want_b), (_, o, o_b) = ref.backward(g64[:, cols], x64[:, ks], held[:, cols], w64[cols][:, ks], act, t)
        ref.within(dw[cols.cuda()][:, ks.cuda()], want, o, ("dw", act))
        ref.within(db[cols.cuda()], want_b, o_b, ("db", act))


@pytest.mark.parametrize("dtype", DTYPES)
def test_weight_gradient_from_codes(dtype):
    """Long contractions over rows whose inputs are 8-bit codes (three bf16 products a value in f32)."""
    lin, t = linear(), DTYPES[dtype]
    for M, K, N in ((4100, 264, 520), (2047, 1000, 130), (300, 2056, 2048)):
        x, w, b, r, g = inputs(M, K, N, t, 5 * M)
        held = lin.tv_checkpoint8(x)
        x64 = held.restore().double().cpu()
        dx, dw, db = lin.tv_linear_backward(g, held, None, w, bias_grad=True)
        rows, cols, ks = sample(M), sample(N), sample(K)
        (_, want, want_b), (_, o, o_b) = ref.backward(g.double().cpu()[:, cols], x64[:, ks], torch.zeros(M, len(cols), dtype=torch.float64),
                                                      w.double().cpu()[cols][:, ks], "none", t)
        ref.within(dw[cols.cuda()][:, ks.cuda()], want, o, "dw")
        ref.within(db[cols.cuda()], want_b, o_b, "db")


def test_more_than_32_bits_of_offsets():
    """x, dx and y of more than 2^31 elements and 2^32 bytes: the last rows are right."""
    lin = linear()
    for t, K, N in ((torch.bfloat16, 1024, 40), (torch.bfloat16, 40, 1024)):
        M = (1 << 31) // 1024 + 777
        gen = torch.Generator(device="cuda").manual_seed(9)
        x = torch.empty(M, K, dtype=t, device="cuda").normal_(generator=gen)
        w = (torch.randn(N, K, generator=gen, device="cuda") * K ** -0.5).to(t)
        y = lin.tv_linear(x, w, act="silu")
        tail = torch.cat([torch.arange(5), torch.arange(M - 300, M)])
        x64, w64 = x[tail.cuda()].double().cpu(), w.double().cpu()
        _, y64, _, off = ref.forward(x64, w64, None, None, "silu", t)
        ref.within(y[tail.cuda()], y64, off, "y")
        del y
        g = torch.empty(M, N, dtype=t, device="cuda").normal_(generator=gen)
        dx = lin._backward(g, None, None, K, None, None, w, K, "none", (True, False, False))[0]
        want, off = ref.backward(g[tail.cuda()].double().cpu(), x64, torch.zeros(len(tail), N, dtype=torch.float64), w64, "none", t)
        ref.within(dx[tail.cuda()], want[0], off[0], "dx")
        del dx
        # dW sums over all rows: exact for small whole numbers (2^31 / 1024 ones, each row's product a one)
        g.zero_()
        g[::7, 0] = 1.0
        x.zero_()
        x[::7, K - 1] = 1.0
        dw = lin._backward(g, x, None, K, None, None, w, K, "none", (False, True, False))[1]
        count = (M + 6) // 7
        assert abs(float(dw[0, K - 1]) - count) <= count * 2.0 ** -8 and float(dw.float().abs().sum()) == float(dw[0, K - 1])


def test_infinities_and_nans_in_large_f32_products():
    """What f32 products give next to infinities, NaNs and the largest numbers, from bf16 parts."""
    lin = linear()
    M, K, N = 300, 520, 260
    x, w, _, _, _ = inputs(M, K, N, torch.float32, 3)
    x[5, 7], x[17, 500], x[33, 0], x[290, 519] = float("inf"), float("-inf"), float("nan"), 3.4e38
    w[0, 7], w[3, 7] = 0.0, 1.0                     # infinity times zero, and times a value with nothing past its first part
    w[:, 519] = 0.5
    y = lin.tv_linear(x, w).double().cpu()
    want = x.double().cpu() @ w.double().cpu().T
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(y), torch.isnan(want)) and torch.equal(torch.isinf(y), torch.isinf(want))
    assert torch.equal(y[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    size = x.double().cpu().abs().nan_to_num(posinf=0.0) @ w.double().cpu().abs().T
    assert ((y - want).abs()[fine] <= ((K + 8) * ref.U32 * size + 1e-38)[fine]).all()
