"""8-bit checkpoints on the GPU: codes and bytes equal to the definition's, exactly."""
import numpy as np
import pytest
import torch

import linref as ref

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def linear():
    from paper_2204_03643_amd import linear as module
    return module


def check(x):
    held = linear().tv_checkpoint8(x)
    v = x.detach().double().cpu().numpy().reshape(-1, x.shape[-1])
    codes, exps = ref.checkpoint8(v)
    assert held.codes.shape == x.shape
    assert np.array_equal(held.exps.cpu().numpy(), exps)
    assert np.array_equal(held.codes.cpu().numpy().reshape(v.shape), codes)
    want = ref.restored(codes, exps)
    got = held.restore()
    assert got.dtype == x.dtype and got.shape == x.shape
    assert np.array_equal(got.double().cpu().numpy().reshape(v.shape), want, equal_nan=True)
    return held


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 40), (7, 1001), (64, 96), (130, 256), (1, 100000), (1000, 8)])
def test_codes_are_the_definitions(rows, n, dtype):
    gen = torch.Generator().manual_seed(rows * 1000 + n)
    x = torch.randn(rows, n, generator=gen) * torch.exp2(torch.randint(-20, 20, (rows, n), generator=gen).float())
    check(x.to(DTYPES[dtype]).cuda())
    x = torch.randn(rows, n, generator=gen)                    # many ties in bf16
    check(x.to(DTYPES[dtype]).cuda())


def test_ends_of_the_range():
    rows = [[0.0] * 32, [-0.0] * 32, [2.0 ** -149] * 32, [2.0 ** -126] * 32, [2.0 ** -120] * 32, [1.5 * 2.0 ** -120, 2.0 ** -127] * 16,
            [3.4028234e38, -3.4028234e38] * 16, [127.5, 127.49, -127.5, 1.0] * 8, [0.5, 1.5, 2.5, -0.5, -1.5, 64.0, 63.5, 62.5] * 4,
            [float("inf"), 1.0, -3.0, float("nan")] * 8, [float("nan")] * 32, [float("-inf")] * 32, [1.0] * 31 + [float("inf")]]
    x = torch.tensor(rows, dtype=torch.float32)
    check(x.cuda())
    check(x.bfloat16().cuda())
    check(x[:, :7].cuda())                                     # rows that are not dense
    held = linear().tv_checkpoint8(x.cuda())
    assert not torch.isnan(held.restore()[9, 1:3]).any()       # what is finite beside a NaN stays


def test_strides_offsets_and_leading_axes():
    gen = torch.Generator().manual_seed(5)
    big = torch.full((40, 300), float("nan"))
    big[2:35, 3:260] = torch.randn(33, 257, generator=gen)
    for t in DTYPES.values():
        b = big.to(t).cuda()
        check(b[2:35, 3:260])
        check(b[2:35, 4:260])
        check(b[2:35, 8:72])
        check(b[2:35:2, 8:72])
        check(b[2:35, 8:72].t())
        check(torch.randn(2, 3, 5, 48, generator=gen).to(t).cuda())
        assert linear().tv_checkpoint8(torch.empty(0, 7, dtype=t, device="cuda")).restore().shape == (0, 7)


def test_a_checkpoint_of_a_checkpoint_is_itself():
    held = linear().tv_checkpoint8(torch.randn(50, 333, device="cuda"))
    again = linear().tv_checkpoint8(held.restore())
    assert torch.equal(held.restore(), again.restore())
    assert held.nbytes == 50 * 333 + 50 * 11


def test_offsets_beyond_32_bits():
    """More than 2^32 samples in one tensor: the last rows are right."""
    rows, n = (1 << 32) // 4096 + 3, 4096
    x = torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(4, n, generator=torch.Generator().manual_seed(1)).bfloat16()
    x[-4:] = tail.cuda()
    held = linear().tv_checkpoint8(x)
    codes, exps = ref.checkpoint8(tail.double().numpy())
    assert np.array_equal(held.codes[-4:].cpu().numpy(), codes) and np.array_equal(held.exps[-4:].cpu().numpy(), exps)
    assert np.array_equal(held.restore()[-4:].double().cpu().numpy(), ref.restored(codes, exps))
