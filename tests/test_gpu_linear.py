"""Channel products and their gradients on the GPU against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import linref as ref

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu", "silu")
# one token, few tokens, tiles that end early in every direction, long contractions with few outputs and the reverse
SHAPES = [(1, 1, 1), (1, 32, 32), (1, 4096, 96), (3, 33, 31), (7, 1001, 777), (16, 520, 264), (17, 64, 5), (33, 8, 2000),
          (64, 2048, 128), (129, 130, 131), (200, 96, 1), (256, 512, 512), (300, 1, 70), (513, 72, 520), (640, 1280, 384)]


def linear():
    from paper_2204_03643_amd import linear as module
    return module


def draw(shape, dtype, seed, scale=1.0):
    """(GPU tensor, the same values in f64 on the CPU)."""
    t = (torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * scale).to(dtype)
    return t.cuda(), t.double()


def inputs(M, K, N, dtype, seed=0):
    x, x64 = draw((M, K), dtype, seed + 1)
    w, w64 = draw((N, K), dtype, seed + 2, K ** -0.5)
    b, b64 = draw((N,), dtype, seed + 3)
    r, r64 = draw((M, N), dtype, seed + 4)
    g, g64 = draw((M, N), dtype, seed + 5)
    return (x, w, b, r, g), (x64, w64, b64, r64, g64)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_forward(M, K, N, dtype):
    lin, t = linear(), DTYPES[dtype]
    (x, w, b, r, _), (x64, w64, b64, r64, _) = inputs(M, K, N, t)
    for act in ACTS:
        for bias, residual in ((True, True), (False, False)):
            y = lin.tv_linear(x, w, b if bias else None, r if residual else None, act)
            _, y64, _, off = ref.forward(x64, w64, b64 if bias else None, r64 if residual else None, act, t)
            ref.within(y, y64, off, (act, bias, residual))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_backward_from_what_is_held(M, K, N, dtype):
    """The gradients alone, from z and x as they are and from 8-bit codes of both."""
    lin, t = linear(), DTYPES[dtype]
    (x, w, _, _, g), (x64, w64, _, _, g64) = inputs(M, K, N, t, 10)
    z, z64 = draw((M, N), t, 99, 2.0)
    x8, z8 = lin.tv_checkpoint8(x), lin.tv_checkpoint8(z)
    xr = torch.from_numpy(ref.restored(*ref.checkpoint8(x64.numpy())))
    zr = torch.from_numpy(ref.restored(*ref.checkpoint8(z64.numpy())))
    words = torch.from_numpy(ref.bits(z64.numpy())).cuda()
    for act in ACTS:
        for held in ("full", "8bit"):
            hz = {"none": None, "relu": words}.get(act, z if held == "full" else z8)
            hz64 = z64 if act == "relu" or held == "full" else zr
            got = lin.tv_linear_backward(g, x if held == "full" else x8, hz, w, act, bias_grad=True)
            want, off = ref.backward(g64, x64 if held == "full" else xr, hz64, w64, act, t)
            for name, a, b, o in zip(("dx", "dw", "db"), got, want, off):
                ref.within(a, b, o, (act, held, name))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("checkpoint", ("full", "8bit"))
@pytest.mark.parametrize("act", ACTS)
def test_autograd_holds_what_it_says(act, checkpoint, dtype):
    """Forward and backward through autograd.  The gradients belong to x and z as held: z is re-made here from the
    codes' definition, off by a step of its block at most."""
    lin, t = linear(), DTYPES[dtype]
    M, K, N = 70, 200, 130
    (x, w, b, r, g), (x64, w64, b64, r64, g64) = inputs(M, K, N, t, 20)
    leaves = [v.clone().requires_grad_() for v in (x, w, b, r)]
    y = lin.tv_linear(*leaves, act=act, checkpoint=checkpoint)
    plain = lin.tv_linear(x, w, b, r, act=act)
    assert torch.equal(y, plain)                              # holding z changes no bit of y
    got = torch.autograd.grad(y, leaves, g)
    z64, _, z_off, _ = ref.forward(x64, w64, b64, None, act, t)
    hx, dz_doubt = x64, torch.zeros_like(z64)
    if act == "relu":                                         # a sign within rounding of zero may be either
        dz_doubt = torch.where(z64.abs() <= z_off, g64.abs(), 0.0)
    if checkpoint == "8bit":
        hx = torch.from_numpy(ref.restored(*ref.checkpoint8(x64.numpy())))
    if act in ("gelu", "silu"):                               # |act''| <= 0.8
        codes, exps = ref.checkpoint8(z64.numpy())
        step = torch.from_numpy(np.ldexp(1.0, np.repeat(exps.astype(int) - 127, 32, 1)[:, :N]))
        rounding = step if checkpoint == "8bit" else ref.unit(t) * z64.abs()
        dz_doubt = 0.8 * g64.abs() * (z_off + rounding)
    want, off = ref.backward(g64, hx, z64, w64, act, t)
    off = (off[0] + dz_doubt @ w64.abs() * 1.01, off[1] + dz_doubt.T @ hx.abs() * 1.01, off[2] + dz_doubt.sum(0) * 1.01)
    for name, a, v, o in zip(("dx", "dw", "db"), got, want, off):
        ref.within(a, v, o, name)
    assert torch.equal(got[3], g)


def test_z_in_8_bits_from_the_epilogue():
    """The codes that the forward call writes stand for z to within their definition's rounding."""
    import paper_2204_03643_amd as tv
    for t, M, K, N in ((torch.bfloat16, 37, 64, 100), (torch.float32, 300, 700, 33), (torch.bfloat16, 5, 2048, 640)):
        (x, w, b, _, _), (x64, w64, b64, _, _) = inputs(M, K, N, t, 30)
        y = torch.empty(M, N, dtype=t, device="cuda")
        codes = torch.full((M, N), 99, dtype=torch.int8, device="cuda")
        exps = torch.full((M, -(-N // 32)), 99, dtype=torch.uint8, device="cuda")
        desc = tv.tv_linear_desc(M, K, N, K, K, N, N, tv.TV_BF16 if t == torch.bfloat16 else tv.TV_F32, tv.TV_ACT_SILU)
        nbytes = tv.tv_linear_fwd_workspace_bytes(desc)
        ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
        held = tv.tv_held(codes.data_ptr(), exps.data_ptr(), tv.TV_HELD_8BIT)
        tv.tv_linear_fwd(x, w, b, None, y, held, desc, ws, nbytes)
        z64, _, z_off, _ = ref.forward(x64, w64, b64, None, "silu", t)
        got = torch.from_numpy(ref.restored(codes.cpu().numpy(), exps.cpu().numpy()))
        step = torch.from_numpy(np.ldexp(1.0, np.repeat(exps.cpu().numpy().astype(int) - 127, 32, 1)[:, :N]))
        clamped = codes.cpu().abs() == 127
        ref.within(got, z64, z_off + step * torch.where(clamped, 1.0, 0.5), (t, M, K, N))
        top = torch.nn.functional.pad(z64.abs(), (0, -N % 32)).view(M, -1, 32).amax(-1)
        assert (step[:, ::32] <= top / 64 * 1.0001).all() and (step[:, ::32] * 128 >= top * 0.9999).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_against_differences(dtype):
    """<grad, d> against (f(p + hd) - f(p - hd)) / 2h of the kernels' own f32 forward pass, f = <g, y>."""
    lin, t = linear(), torch.float32
    M, K, N = 40, 56, 72
    (x, w, b, r, g), _ = inputs(M, K, N, t, 40)
    if dtype == "bf16":                                       # values that bf16 holds, so that both paths see the same
        x, w, b, r, g = (v.bfloat16().float() for v in (x, w, b, r, g))
    for act in ("none", "gelu", "silu"):
        leaves = [v.to(DTYPES[dtype]).requires_grad_() for v in (x, w, b, r)]
        grads = torch.autograd.grad(lin.tv_linear(*leaves, act=act), leaves, g.to(DTYPES[dtype]))
        for i, grad in enumerate(grads):
            d = draw(tuple(grad.shape), t, 50 + i)[0]
            h = 2.0 ** -6
            up, down = [x, w, b, r], [x, w, b, r]
            up[i], down[i] = up[i] + h * d, down[i] - h * d
            diff = (lin.tv_linear(*up, act=act) - lin.tv_linear(*down, act=act)).double()
            want = float((g.double() * diff.detach()).sum() / (2 * h))
            got = float((grad.double() * d.double()).sum())
            # f32 outputs of size about 2 are off by 2^-21 each, divided by 2h and summed with signs at random; the
            # third derivatives (at most 2, times (h d . x)^3 / 6 with d . x of size sqrt(K) at most) and the
            # gradients' own rounding (2^-8 or 2^-24 of each term) come on top
            noise = float(g.double().norm()) * 2.0 ** -21 / (2 * h) * 4
            cubic = h * h / 6 * 2 * float((g.double().abs()).sum()) * (0.0 if act == "none" else 15.0)
            rounding = 4 * ref.unit(DTYPES[dtype]) * 3 * float((grad.double() * d.double()).norm())
            assert abs(got - want) <= noise + cubic + rounding, (act, i, got, want, noise, cubic, rounding)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [(5, 37, 41), (130, 264, 136), (300, 520, 257), (16, 1024, 64)])
def test_strides_and_surroundings(M, K, N, dtype):
    """Rows inside larger arrays that hold NaN around them, at odd addresses: nothing is read or written outside."""
    import paper_2204_03643_amd as tv
    lin, t = linear(), DTYPES[dtype]
    (x, w, b, r, g), (x64, w64, b64, r64, g64) = inputs(M, K, N, t, 60)

    def inside(v, before, after):
        big = torch.full((v.shape[0] + 2, v.shape[1] + before + after), float("nan"), dtype=v.dtype, device="cuda")
        big[1:-1, before:before + v.shape[1]] = v
        return big, big[1:-1, before:before + v.shape[1]]

    for before, after in ((0, 8), (1, 2), (3, 0)):
        xs, ws_, rs, gs = (inside(v, before, after)[1] for v in (x, w, r, g))
        y = lin.tv_linear(xs, ws_, b, rs, "silu")
        _, y64, _, off = ref.forward(x64, w64, b64, r64, "silu", t)
        ref.within(y, y64, off, "y")
        z, z64 = draw((M, N), t, 70)
        got = lin.tv_linear_backward(gs, xs, z, ws_, "gelu", bias_grad=True)
        want, off3 = ref.backward(g64, x64, z64, w64, "gelu", t)
        for name, a, v, o in zip(("dx", "dw", "db"), got, want, off3):
            ref.within(a, v, o, name)
        # y inside a larger array, its surroundings untouched
        big, ys = inside(torch.zeros(M, N, dtype=t, device="cuda"), before, after)
        marks = torch.isnan(big).clone()
        desc = tv.tv_linear_desc(M, K, N, xs.stride(0), ws_.stride(0), rs.stride(0), ys.stride(0),
                                 tv.TV_BF16 if t == torch.bfloat16 else tv.TV_F32, tv.TV_ACT_SILU)
        nbytes = tv.tv_linear_fwd_workspace_bytes(desc)
        ws = torch.full((max(nbytes, 16),), 255, dtype=torch.uint8, device="cuda")     # NaN for whoever reads it
        tv.tv_linear_fwd(xs, ws_, b, rs, ys, tv.tv_held(None, None, 0), desc, ws, nbytes)
        ref.within(ys, y64, off, "y inside")
        assert torch.equal(torch.isnan(big), marks)
        ys.copy_(rs)                                          # y may be the residual itself
        tv.tv_linear_fwd(xs, ws_, b, ys, ys, tv.tv_held(None, None, 0), desc, ws, nbytes)
        assert torch.equal(ys, y)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K,N", [(4, 256, 64), (200, 300, 136), (257, 1024, 256)])
def test_non_finite_values_stay_in_their_rows(M, K, N, dtype):
    lin, t = linear(), DTYPES[dtype]
    (x, w, b, _, g), _ = inputs(M, K, N, t, 80)
    clean = lin.tv_linear(x, w, b, act="silu")
    bad = x.clone()
    bad[1, K // 2], bad[3, 0] = float("inf"), float("nan")
    y = lin.tv_linear(bad, w, b, act="silu")
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[1] = rows[3] = False
    assert torch.equal(y[rows], clean[rows]) and torch.isnan(y[3]).all()
    # infinity times a weight that is not zero; silu of -infinity is infinity times zero
    toward = w[:, K // 2].float()
    assert torch.isposinf(y[1][toward > 0]).all() and torch.isnan(y[1][toward < 0]).all()
    z = torch.randn(M, N, device="cuda").to(t)
    dx, dw, db = lin.tv_linear_backward(g, bad, z, w, "gelu", True)
    dx0, dw0, db0 = lin.tv_linear_backward(g, x, z, w, "gelu", True)
    assert torch.equal(dx, dx0) and torch.equal(db, db0)
    cols = torch.ones(K, dtype=torch.bool, device="cuda")
    cols[K // 2] = cols[0] = False
    assert torch.equal(dw[:, cols], dw0[:, cols]) and torch.isnan(dw[:, 0]).all()


def test_masked_gradients_do_not_reach_relu():
    """Where ReLU is off, an infinite or NaN gradient does not come through."""
    lin = linear()
    M, N, K = 33, 70, 40
    (x, w, _, _, g), _ = inputs(M, K, N, torch.float32, 90)
    z = torch.randn(M, N, generator=torch.Generator().manual_seed(3))
    z[2, 5], z[7, 64] = -1.0, -1.0
    g[2, 5], g[7, 64] = float("inf"), float("nan")
    words = torch.from_numpy(ref.bits(z.double().numpy())).cuda()
    got = lin.tv_linear_backward(g, x, words, w, "relu", True)
    g0 = g.clone()
    g0[2, 5] = g0[7, 64] = 0.0
    for a, b in zip(got, lin.tv_linear_backward(g0, x, words, w, "relu", True)):
        assert torch.isfinite(a).all() and torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_rows(dtype):
    lin, t = linear(), DTYPES[dtype]
    w = torch.randn(6, 9, device="cuda").to(t).requires_grad_()
    b = torch.randn(6, device="cuda").to(t).requires_grad_()
    x = torch.empty(2, 0, 9, dtype=t, device="cuda", requires_grad=True)
    for checkpoint in ("full", "8bit"):
        y = lin.tv_linear(x, w, b, act="gelu", checkpoint=checkpoint)
        assert y.shape == (2, 0, 6)
        dx, dw, db = torch.autograd.grad(y, (x, w, b), torch.empty_like(y))
        assert dx.shape == x.shape and not dw.any() and not db.any()


def test_leading_axes_views_and_frozen_parameters():
    lin = linear()
    x = torch.randn(3, 5, 64, device="cuda")
    w, b = torch.randn(48, 64, device="cuda"), torch.randn(48, device="cuda")
    r = torch.randn(5, 48, device="cuda").expand(3, 5, 48)
    y = lin.tv_linear(x, w, b, r, "silu")
    flat = lin.tv_linear(x.reshape(15, 64), w, b, r.reshape(15, 48), "silu")
    assert torch.equal(y.reshape(15, 48), flat)
    assert torch.equal(lin.tv_linear(x.transpose(0, 1), w, b, None, "silu"),
                       lin.tv_linear(x.transpose(0, 1).contiguous(), w, b, None, "silu"))
    wt = torch.randn(64, 48, device="cuda")
    assert torch.equal(lin.tv_linear(x, wt.t(), b), lin.tv_linear(x, wt.t().contiguous(), b))
    xg = x.clone().requires_grad_()
    yg = lin.tv_linear(xg, w, b, None, "gelu", "8bit")
    assert yg.grad_fn.saved_tensors[0] is None                # a frozen weight: x is not held
    (dx,) = torch.autograd.grad(yg.sum(), xg)
    assert dx.shape == x.shape
    bg = b.clone().requires_grad_()
    (db,) = torch.autograd.grad(lin.tv_linear(x, w, bg, None, "none"), bg, torch.ones(3, 5, 48, device="cuda"))
    assert torch.allclose(db, torch.full_like(db, 15.0))


def test_same_bits_every_time_on_any_stream():
    lin = linear()
    for t, M, K, N in ((torch.bfloat16, 100, 4096, 96), (torch.float32, 300, 600, 200), (torch.bfloat16, 1024, 512, 512)):
        (x, w, b, r, g), _ = inputs(M, K, N, t, 100)
        leaves = [v.requires_grad_() for v in (x, w, b, r)]

        def both():
            y = lin.tv_linear(*leaves, act="gelu", checkpoint="8bit")
            return (y.detach(),) + torch.autograd.grad(y, leaves, g)
        first = both()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            again = both()
        side.synchronize()
        for a, b_ in zip(first, again):
            assert torch.equal(a, b_)


def test_graph_capture_and_replays():
    lin = linear()
    for t, M, K, N in ((torch.bfloat16, 1, 1024, 512), (torch.bfloat16, 256, 1024, 512), (torch.float32, 130, 700, 96)):
        (x, w, b, r, g), _ = inputs(M, K, N, t, 110)
        z = torch.randn(M, N, device="cuda").to(t)

        def step():
            held = lin.tv_checkpoint8(x)
            return (lin.tv_linear(x, w, b, r, "gelu"),) + lin.tv_linear_backward(g, held, z, w, "gelu", True)
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        for i in range(3):
            x.copy_(torch.randn(M, K, device="cuda").to(t))
            want = step()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for a, v in zip(out, want):
                assert torch.equal(a, v), i
