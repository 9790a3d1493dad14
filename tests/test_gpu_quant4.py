"""Values in 4 bits and products of them, against their definition."""
import linref
import numpy as np
import pytest
import quant4ref
import torch

pytestmark = pytest.mark.gpu


def held(x):
    """A Quantized4 and what the definition says, compared."""
    from paper_2204_03643_amd.quant4 import tv_quantize4
    q = tv_quantize4(x)
    rows = x.reshape(-1, x.shape[-1])
    codes, exps = quant4ref.save(rows.double().cpu().numpy())
    assert q.codes.cpu().numpy().tolist() == codes.tolist()
    assert np.array_equal(q.exps.cpu().numpy(), exps)
    got = q.restore()
    assert got.shape == x.shape and got.dtype == x.dtype
    want = quant4ref.load(codes, exps, x.shape[-1])
    assert np.array_equal(got.double().cpu().numpy().reshape(rows.shape), want, equal_nan=True)
    return q


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 31), (2, 32), (3, 33), (5, 127), (4, 128), (17, 129), (7, 300), (16, 256), (33, 1001), (1, 8192), (70, 64)])
def test_values(rows, n, dtype):
    gen = torch.Generator().manual_seed(rows * 7 + n)
    held((torch.randn(rows, n, generator=gen) * torch.exp2(torch.randint(-30, 30, (rows, 1), generator=gen))).to(dtype).cuda())


def test_values_at_the_borders():
    """Each border between two values and its neighbours on either side, with all the scales of f32 there are."""
    lines = []
    for e in (-122, -121, -60, -1, 0, 1, 60, 124, 125):
        at = []
        for b, _ in quant4ref.BORDERS + ((4.0, 0), (6.0, 0), (7.0, 0), (7.999, 0)):
            f = np.float32(np.ldexp(np.float32(b), e))
            at += [f, np.nextafter(f, np.float32(0)), np.nextafter(f, np.float32(np.inf))]
        at = np.array(at, np.float32)
        at = at[np.abs(at) < np.ldexp(8.0, e)]
        line = np.zeros(128, np.float32)
        for i, v in enumerate(at):
            line[i % 31 + 32 * (i // 31)] = v if i % 2 else -v
        line[31::32] = np.ldexp(np.float32(4.0), e)
        lines.append(line)
    held(torch.from_numpy(np.stack(lines)).cuda())


def test_every_bf16():
    bits = torch.arange(1 << 16, dtype=torch.int32) << 16
    held(bits.view(torch.float32).to(torch.bfloat16).view(-1, 512).cuda())


def test_blocks_that_are_not_finite():
    x = torch.randn(6, 100)
    x[0, 5], x[1, 40], x[2, 99], x[3, 96] = float("nan"), float("inf"), float("-inf"), float("nan")
    back = held(x.cuda()).restore().cpu()
    spoiled = back.isnan()
    assert spoiled[0, :32].all() and spoiled[1, 32:64].all() and spoiled[2, 96:].all() and spoiled[3, 96:].all()
    assert int(spoiled.sum()) == 32 + 32 + 4 + 4


def test_small_and_large_values():
    x = torch.tensor([[1e-45, 1e-40, 0.0, -0.0], [2.0 ** -120, 2.0 ** -123, 2.0 ** -126, 0.0], [3.4e38, 1e38, -2e37, 1.0]])
    held(x.cuda())
    held(torch.zeros(3, 40, device="cuda"))


def test_views():
    from paper_2204_03643_amd.quant4 import tv_quantize4
    base = torch.randn(20, 500, device="cuda")
    for v in (base[:, 3:290], base.t(), base[::2, 1:], base.view(4, 5, 500), base[0]):
        a, b = tv_quantize4(v), tv_quantize4(v.contiguous())
        assert torch.equal(a.codes, b.codes) and torch.equal(a.exps, b.exps) and torch.equal(a.restore(), b.restore())


def test_views_that_stand_for_the_negative_of_their_memory():
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    for n in (1, 40):
        z = torch.randn(3, n, dtype=torch.complex64, device="cuda")
        v = z.conj().imag
        assert v.is_neg() and torch.equal(tv_quantize4(v).restore(), tv_quantize4(v.resolve_neg().clone()).restore())
        w = tv_quantize4(torch.randn(n, n, device="cuda"))
        for m in (1, 3):
            want = tv_linear4(v[:m].resolve_neg().clone(), w, v[0].resolve_neg().clone(), v[:m].resolve_neg().clone())
            assert torch.equal(tv_linear4(v[:m], w, v[0], v[:m]), want)


def test_many_rows_and_groups():
    """More rows and more groups than a launch's workgroups."""
    from paper_2204_03643_amd.quant4 import tv_quantize4
    for rows, n in (((1 << 20) + 37, 24), (3, 256 * 128 * 3 + 5)):
        x = torch.randn(rows, n, device="cuda")
        q = tv_quantize4(x)
        some = torch.tensor([0, 1, rows // 2, rows - 1], device="cuda")
        codes, exps = quant4ref.save(x[some].double().cpu().numpy())
        assert np.array_equal(q.codes[some].cpu().numpy(), codes) and np.array_equal(q.exps[:, some].cpu().numpy(), exps[:, :4])
        assert np.array_equal(q.restore()[some].double().cpu().numpy(), quant4ref.load(codes, exps, n))


def product(M, K, N, dtype, act, bias, residual, seed=0, lead=None):
    gen = torch.Generator().manual_seed(seed + M + K + N)
    x = (torch.randn(M, K, generator=gen) * torch.exp2(torch.randn(M, 1, generator=gen))).to(dtype)
    w = torch.randn(N, K, generator=gen).to(dtype) / K ** 0.5
    b = torch.randn(N, generator=gen).to(dtype) if bias else None
    r = torch.randn(M, N, generator=gen).to(dtype) if residual else None
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    c = [None if t is None else t.cuda() for t in (x, w, b, r)]
    w4 = tv_quantize4(c[1])
    got = tv_linear4(c[0], w4, c[2], c[3], act=act)
    assert torch.equal(tv_linear4(tv_quantize4(c[0]), w4, c[2], c[3], act=act), got)
    stands = [torch.from_numpy(quant4ref.load(*quant4ref.save(t.double().numpy()), K)) for t in (x, w)]
    wide = [None if t is None else t.double() for t in (b, r)]
    _, y, _, off = linref.forward(*stands, *wide, act, dtype)
    linref.within(got, y, off, "y")
    return got


SHAPES = [(1, 1, 1), (1, 32, 16), (1, 2048, 512), (2, 100, 33), (7, 1001, 777), (16, 128, 64), (17, 129, 65), (31, 300, 100), (33, 4096, 48),
          (64, 640, 200), (65, 256, 128), (100, 512, 130), (129, 1000, 257), (200, 64, 300), (256, 2048, 256), (257, 384, 515), (600, 896, 1030), (3, 130, 4104), (16, 2048, 4100), (29, 257, 8192), (1, 1000, 8200),
          (17, 300, 8200), (2, 8200, 100)]


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("M,K,N", SHAPES)
def test_products(M, K, N, dtype):
    product(M, K, N, dtype, "none", False, False)
    product(M, K, N, dtype, "gelu", True, True, seed=1)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("act", ("none", "relu", "gelu", "silu"))
def test_epilogues(act, dtype):
    for bias, residual in ((True, False), (False, True), (True, True)):
        product(70, 200, 90, dtype, act, bias, residual, seed=3)


# products through each size of tile, with last tiles that are not whole, and split contractions that are joined
LARGE = [(2049, 1100, 4100), (4097, 2304, 4104), (1500, 1300, 2100), (4100, 257, 4100), (300, 5000, 500), (70, 4100, 300), (129, 8200, 1001)]


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16))
@pytest.mark.parametrize("M,K,N", LARGE)
def test_large_products(M, K, N, dtype):
    """Against products of the restored values in 64 bits on the GPU (restoring is held to its definition above)."""
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    x, w, r = (torch.randn(*s, generator=gen, device="cuda").to(dtype) for s in ((M, K), (N, K), (M, N)))
    b = torch.randn(N, generator=gen, device="cuda").to(dtype)
    x4, w4 = tv_quantize4(x * 2), tv_quantize4(w / K ** 0.5)
    wide = x4.restore().double(), w4.restore().double(), b.double(), r.double()
    for act, bias, residual in (("none", False, False), ("gelu", True, True), ("silu", True, False)):
        got = tv_linear4(x4, w4, b if bias else None, r if residual else None, act=act)
        _, y, _, off = linref.forward(*wide[:2], wide[2] if bias else None, wide[3] if residual else None, act, dtype)
        assert bool(((got.double() - y).abs() <= off).all()), (act, float(((got.double() - y).abs() - off).max()))
        if act == "none":
            assert torch.equal(tv_linear4(x * 2, w4), got)


@pytest.mark.parametrize("M", (1, 40, 300))
def test_each_block_has_its_own_scale(M):
    """Scales that differ from block to block by many powers of two, of x and of W, so that a scale taken from a neighbour shows."""
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    gen = torch.Generator().manual_seed(M)
    K, N = 1024, 200
    sx, sw = (torch.exp2(torch.randint(-8, 8, (r, K // 32, 1), generator=gen).double()) for r in (M, N))
    x = (torch.randn(M, K // 32, 32, generator=gen).double() * sx).view(M, K)
    w = (torch.randn(N, K // 32, 32, generator=gen).double() / sx[:1].repeat(N, 1, 1) * sw).view(N, K)
    got = tv_linear4(x.float().cuda(), tv_quantize4(w.float().cuda()))
    x4, w4 = (torch.from_numpy(quant4ref.load(*quant4ref.save(t.float().numpy()), K)) for t in (x, w))
    _, y, _, off = linref.forward(x4, w4, None, None, "none", torch.float32)
    linref.within(got, y, off, "y")


@pytest.mark.parametrize("M", (3, 90, 260))
def test_a_row_that_is_not_finite_stays_by_itself(M):
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    x, w = torch.randn(M, 333, device="cuda"), torch.randn(140, 333, device="cuda")
    clean = tv_linear4(x, tv_quantize4(w))
    x[1, 332], w[5, 0] = float("inf"), float("nan")
    y = tv_linear4(x, tv_quantize4(w))
    assert y[1].isnan().all() and y[:, 5].isnan().all()
    clean[1], clean[:, 5] = float("nan"), float("nan")
    assert torch.equal(y.nan_to_num(7.0), clean.nan_to_num(7.0))


def test_rows_of_a_product_do_not_depend_on_what_else_is_there():
    """The same values as a view, as a copy and as codes."""
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    w = tv_quantize4(torch.randn(100, 250, device="cuda"))
    base = torch.randn(50, 600, device="cuda").bfloat16()
    r = torch.randn(50, 300, device="cuda").bfloat16()
    y = tv_linear4(base[:, 3:253], w, residual=r[:, 1:101])
    assert torch.equal(tv_linear4(base[:, 3:253].contiguous(), w, residual=r[:, 1:101].contiguous()), y)
    assert torch.equal(tv_linear4(base[:, 3:253].reshape(5, 10, 250), w, residual=r[:, 1:101].reshape(5, 10, 100)).view(50, 100), y)
    assert tv_linear4(base[:0, 3:253], w).shape == (0, 100)
    assert torch.equal(tv_linear4(base[0, 3:253], w, residual=r[0, 1:101]), tv_linear4(base[:1, 3:253], w, residual=r[:1, 1:101])[0])


@pytest.mark.parametrize("M", (2, 50, 300))
def test_captured(M):
    from paper_2204_03643_amd.quant4 import tv_linear4, tv_quantize4
    w = tv_quantize4(torch.randn(160, 700, device="cuda").bfloat16())
    x = torch.randn(M, 700, device="cuda").bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tv_linear4(x, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = tv_linear4(x, w, act="silu")
    for _ in range(3):
        x.copy_(torch.randn(M, 700, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tv_linear4(x, w, act="silu"), y)


def test_module_and_gradients_refused():
    from paper_2204_03643_amd.linear import TVLinear
    from paper_2204_03643_amd.quant4 import TVLinear4, tv_linear4, tv_quantize4
    torch.manual_seed(0)
    linear = TVLinear(200, 70, act="silu", device="cuda", dtype=torch.bfloat16)
    small = TVLinear4.from_linear(linear)
    x = torch.randn(9, 200, device="cuda").bfloat16()
    want = tv_linear4(x, tv_quantize4(linear.weight), linear.bias.detach(), act="silu")
    assert torch.equal(small(x), want)
    other = TVLinear4(200, 70, act="silu", device="cuda", dtype=torch.bfloat16)
    other.load_state_dict(small.state_dict())
    assert torch.equal(other(x), want) and not list(small.parameters())
    with pytest.raises(RuntimeError, match="no gradients"):
        small(x.requires_grad_())
    with torch.no_grad():
        assert torch.equal(small(x), want)
