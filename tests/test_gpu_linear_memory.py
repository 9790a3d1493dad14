"""What the channel products allocate."""
import pytest
import torch

import paper_2204_03643_amd as tv

pytestmark = pytest.mark.gpu


def peak(call):
    """Bytes that a call holds at its most, beyond what there was (in blocks of 512 bytes, and large ones of 2 MiB)."""
    call()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    kept = call()                                      # noqa: F841 (alive until the peak is read)
    return torch.cuda.max_memory_allocated() - before


def test_no_more_than_the_operands_need():
    from paper_2204_03643_amd.linear import tv_linear, tv_linear_backward
    M, K, N, t = 4096, 2048, 4096, torch.bfloat16
    x, w, g = (torch.randn(*s, device="cuda").to(t) for s in ((M, K), (N, K), (M, N)))
    slack = 4 << 20
    assert peak(lambda: tv_linear(x, w)) <= 2 * M * N + slack
    z = torch.randn(M, N, device="cuda").to(t)
    assert peak(lambda: tv_linear_backward(g, x, z, w, "gelu", True)) <= 2 * (M * N + M * K + N * K) + slack
    # off 16-byte boundaries copies are made, and asked for
    off = torch.randn(M * K + 1, device="cuda").to(t)[1:].view(M, K)
    assert torch.equal(tv_linear(off, w), tv_linear(off.clone(), w))


@pytest.mark.parametrize("wanted", ([0], [1], [2], [0, 2], [1, 2]))
@pytest.mark.parametrize("act", ("none", "gelu", "relu"))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
def test_some_of_the_gradients(wanted, act, dtype):
    """Any of dx, dW and db alone has the bits that it has beside the others."""
    from paper_2204_03643_amd.linear import tv_linear
    for M, K, N in ((40, 72, 88), (300, 1001, 130), (1000, 264, 512)):
        x, w, b, g = (torch.randn(*s, device="cuda").to(dtype) for s in ((M, K), (N, K), (N,), (M, N)))
        leaves = [v.clone().requires_grad_() for v in (x, w, b)]
        everything = torch.autograd.grad(tv_linear(*leaves, act=act), leaves, g)
        some = [v.clone().requires_grad_(i in wanted) for i, v in enumerate((x, w, b))]
        got = torch.autograd.grad(tv_linear(*some, act=act), [some[i] for i in wanted], g)
        for i, v in zip(wanted, got):
            assert torch.equal(v, everything[i]), (M, K, N, i)


@pytest.mark.parametrize("checkpoint", ("full", "8bit"))
@pytest.mark.parametrize("act", ("none", "relu", "gelu", "silu"))
def test_nothing_of_z_is_held_for_a_residual_alone(act, checkpoint):
    from paper_2204_03643_amd.linear import tv_linear
    x, w, b, r, g = (torch.randn(*s, device="cuda") for s in ((70, 64), (48, 64), (48,), (70, 48), (70, 48)))
    y = tv_linear(x, w, b, r.requires_grad_(), act=act, checkpoint=checkpoint)
    held = [t for t in y.grad_fn.saved_tensors if t is not None and t.data_ptr() != w.data_ptr()]
    assert held == []
    assert torch.equal(torch.autograd.grad(y, r, g)[0], g)
    # a bias alone needs z
    y = tv_linear(x, w, b.requires_grad_(), act=act, checkpoint=checkpoint)
    assert sum(t is not None for t in y.grad_fn.saved_tensors[1:4]) == {"none": 0, "relu": 1}.get(act, 2 if checkpoint == "8bit" else 1)


@pytest.mark.parametrize("held", ("full", "8bit"))
@pytest.mark.parametrize("act", ("none", "gelu"))
def test_unwanted_gradients_are_not_computed(act, held):
    from paper_2204_03643_amd.linear import tv_checkpoint8, tv_linear_backward
    M, K, N = 2048, 4096, 2048
    x, w, g, z = (torch.randn(*s, device="cuda").bfloat16() for s in ((M, K), (N, K), (M, N), (M, N)))
    x, z = (tv_checkpoint8(x), tv_checkpoint8(z)) if held == "8bit" else (x, z)
    if act == "none":
        z = None
    def call(dx, dw, db):
        return tv_linear_backward(g, x, z, w, act, bias_grad=db, input_grad=dx, weight_grad=dw)
    everything = call(True, True, True)
    outputs, slack = (2 * M * K, 2 * N * K, 2 * N), 4 << 20
    desc = tv.tv_linear_desc(M, K, N, K, K, N, N, tv.TV_BF16, tv.TV_ACT_GELU if act == "gelu" else tv.TV_ACT_NONE)
    for which in ((True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, False, False)):
        for got, full, wanted in zip(call(*which), everything, which):
            assert torch.equal(got, full) if wanted else got is None
        at = [16 if wanted else None for wanted in which]
        scratch = tv.tv_linear_bwd_workspace_bytes_at(16, 16, 16 if held == "8bit" else None, 16, *at, desc) if any(which) else 0
        most = sum(o for o, wanted in zip(outputs, which) if wanted) + scratch
        assert peak(lambda: call(*which)) <= most + slack
