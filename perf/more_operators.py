"""The measured cases of a residual block's borders (norms, gate, scale, dropout, residual), of dropout by itself, and of
values in 4 bits and products of them, as a program calls them around the channel products of a TV block.

Over rows of n channels:

    norm(v) = (v - mu) r w + b,   r = (mean((v - mu)^2) + eps)^-1/2,   mu = mean(v) ("layer") or 0 ("rms")
    y = x + d scale act(gate) norm(f),   h = next norm(y)

gate is [rows, n], or one row for each sequence of T rows; act is none, sigmoid or silu.  d is 0 where a channel of a row is
dropped and 65536 / (65536 - q) where not, q = round(65536 p).  Philox 4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random
numbers: as easy as 1, 2, 3; 2011) with the 64-bit seed as its key gives, for the counter (column / 8, row, offset's low
half, offset's high half), eight numbers of 16 bits, the lower half of each word first; a column is dropped where its number
is below q.

4 bits: blocks of 32 along a row (the last one may be shorter) share a scale 2^(floor(log2 max) - 2), max the block's largest
magnitude (2^-120 at least); a value over its scale is rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their
negatives, halfway cases to the even code, and to 6 beyond.  Two codes lie in a byte, the first in its lower half: sign bit,
two exponent bits, one of the fraction.  A row's codes are padded to whole groups of 128 values; the four scale bytes
(exponent + 127) of a group lie side by side, those of one group of all rows (padded to a multiple of four) one after another.

  kind  "norm"     forward only                       "norm_train"   forward and gradients
        "block"    y (and h where there is a next norm)  "block_train"  forward and gradients
        "drop"     forward and gradient of dropout alone
        "held4"    a tensor into 4 bits and back
        "linear4"  act(q(x) q(W)^T + b) + r, x in 16 or 32 bits and W in 4
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-6


def _norm(name, B, T, n, dtype, norm="rms", bias=False, train=False):
    return _named(name, dict(kind="norm_train" if train else "norm", B=B, T=T, n=n, dtype=dtype, norm=norm, bias=bias))


def _block(name, B, T, n, dtype, norm, next_norm, bias=False, gate="none", act="none", scale=True, p=0.0, train=False):
    return _named(name, dict(kind="block_train" if train else "block", B=B, T=T, n=n, dtype=dtype, norm=norm,
                             next_norm=next_norm, bias=bias, gate=gate, act=act, scale=scale, p=p))


def _plain_case(name, kind, rows, n, dtype, p=0.0):
    return _named(name, dict(kind=kind, B=1, T=rows, n=n, dtype=dtype, p=p))


def _linear(name, M, K, N, dtype, act="none", bias=True, residual=False):
    return _named(name, dict(kind="linear4", M=M, K=K, N=N, dtype=dtype, act=act, bias=bias, residual=residual))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token before a block: latency alone
        _norm("norm_1x2048_rms_bf16", 1, 1, 2048, "bf16"),
        # the norm before a block in a training step on a large batch
        _norm("norm_8192x2048_rms_bf16_train", 8, 1024, 2048, "bf16", train=True),
        # one token each of 64 streams between two blocks: norm after the one, scale, residual, norm before the next
        _block("between_64x2048_rms_rms_bf16", 64, 1, 2048, "bf16", "rms", "rms"),
        # the same border in a training step: a gate for each of 16 sequences, dropout
        _block("between_16x1024x2048_gate_drop_bf16_train", 16, 1024, 2048, "bf16", "rms", "rms", False, "sequence", "none",
               True, 0.1, True),
        # ragged sizes in f32, layer norms with bias, a gate for each token
        _block("between_3x333x1001_layer_sigmoid_f32_train", 3, 333, 1001, "f32", "layer", "layer", True, "token", "sigmoid",
               True, 0.0, True),
        # dropout of a wide layer's activations on a large batch, with its gradient
        _plain_case("drop_8192x8192_bf16", "drop", 8192, 8192, "bf16", 0.1),
        # dropout of a small ragged tensor
        _plain_case("drop_257x1001_f32", "drop", 257, 1001, "f32", 0.25),
        # activations of a layer on a large batch into 4 bits and back
        _plain_case("held4_16384x4096_bf16", "held4", 16384, 4096, "bf16"),
        # a small ragged tensor into 4 bits and back
        _plain_case("held4_257x1001_f32", "held4", 257, 1001, "f32"),
        # one token of one stream through the first product of a channel block: W's bytes, and latency
        _linear("token4_1x2048to8192_gelu_bf16", 1, 2048, 8192, "bf16", "gelu"),
        # one token each of 64 streams through the second product, with the skip connection
        _linear("tokens4_64x8192to2048_res_bf16", 64, 8192, 2048, "bf16", "none", True, True),
        # a large batch of prompts through the first product
        _linear("prompt4_8192x2048to8192_gelu_bf16", 8192, 2048, 8192, "bf16", "gelu"),
    ]


_MOST_BLOCK = 16384 * 2048
_MOST_HELD = 8192 * 8192
_MOST_MACS = 8192 * 2048 * 8192


def _size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    step = rng.choice((1, 1, 8, 64))
    return min(hi, max(lo, n // step * step))


def draw(rng):
    kind = rng.choice(("norm", "norm_train", "block", "block_train", "block_train", "drop", "held4", "linear4", "linear4"))
    dtype = rng.choice(("bf16", "f32"))
    if kind == "linear4":
        while True:
            M, K, N = _size(rng, 1, 16384), _size(rng, 64, 8192), _size(rng, 64, 8192)
            if M * K * N <= _MOST_MACS:
                break
        return _linear(None, M, K, N, dtype, rng.choice(("none", "relu", "gelu", "silu")), rng.random() < 0.75, rng.random() < 0.5)
    if kind in ("drop", "held4"):
        while True:
            rows, n = _size(rng, 1, 16384), _size(rng, 16, 16384)
            if rows * n <= _MOST_HELD:
                break
        return _plain_case(None, kind, rows, n, dtype, rng.choice((0.1, 0.25, 0.5, 0.73)) if kind == "drop" else 0.0)
    while True:
        B, T, n = _size(rng, 1, 64), _size(rng, 1, 4096), _size(rng, 16, 16384)
        if B * T * n <= _MOST_BLOCK:
            break
    train, norm = kind.endswith("train"), rng.choice(("rms", "layer"))
    bias = norm == "layer" and rng.random() < 0.75
    if kind.startswith("norm"):
        return _norm(None, B, T, n, dtype, norm, bias, train)
    gate = rng.choice(("none", "sequence", "token"))
    return _block(None, B, T, n, dtype, rng.choice(("none", norm)), rng.choice(("none", norm, norm)), bias, gate,
                  "none" if gate == "none" else rng.choice(("none", "sigmoid", "silu")), rng.random() < 0.75,
                  rng.choice((0.0, 0.1, 0.3)), train)


def _blocks(n):
    return -(-n // 32)


def prepare(case, seed):
    t = _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def activations(rows, n):
        """A few channels are much larger than the others, and the size differs from token to token."""
        loud = torch.where(torch.rand(n, generator=gen, device="cuda") < 1.0 / 64, 8.0, 1.0)
        return normal(rows, n) * loud * torch.exp2(normal(rows, 1) * 0.5)

    s = {"case": case}
    if case["kind"] == "linear4":
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = activations(M, K).to(t)
        # a trained weight in 4 bits, as a program that serves it holds it
        s["w4"], s["we"] = _packed(normal(N, K) / math.sqrt(2.0 * K))
        s["b"] = (normal(N) * 0.2).to(t) if case["bias"] else None
        s["r"] = normal(M, N).to(t) if case["residual"] else None
        return s
    B, T, n = case["B"], case["T"], case["n"]
    shape = (B, T, n)
    s["x"] = activations(B * T, n).to(t).view(shape)
    if case["kind"] == "held4":
        return s
    # (the numbers of dropout come from the seed that the program hands over)
    s["seed"], s["offset"] = (int(seed) * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), 7
    leaves = ["x"]
    if case["kind"] == "drop":
        s["gy"] = normal(*shape).to(t)
    elif case["kind"].startswith("norm"):
        s["nw"] = (1.0 + 0.2 * normal(n)).to(t)
        s["nb"] = (0.2 * normal(n)).to(t) if case["bias"] else None
        leaves += ["nw", "nb"]
        if case["kind"] == "norm_train":
            s["gh"] = normal(*shape).to(t)
    else:
        s["f"] = activations(B * T, n).to(t).view(shape)
        affine, after = case["norm"] != "none", case["next_norm"] != "none"
        s["w"] = (1.0 + 0.2 * normal(n)).to(t) if affine else None
        s["b"] = (0.2 * normal(n)).to(t) if affine and case["bias"] else None
        s["nw"] = (1.0 + 0.2 * normal(n)).to(t) if after else None
        s["nb"] = (0.2 * normal(n)).to(t) if after and case["bias"] else None
        s["scale"] = (0.5 + 0.1 * normal(n)).to(t) if case["scale"] else None
        s["gate"] = None if case["gate"] == "none" else normal(B, 1 if case["gate"] == "sequence" else T, n).to(t)
        leaves += ["f", "gate", "scale", "w", "b", "nw", "nb"]
        if case["kind"] == "block_train":
            s["gy"] = normal(*shape).to(t)
            s["gh"] = normal(*shape).to(t) if after else None
    if case["kind"] in ("norm_train", "block_train", "drop"):
        s["leaves"] = [k for k in leaves if s.get(k) is not None]
        for k in s["leaves"]:
            s[k].requires_grad_()
    return s


def _power_of_two(e):
    """2^e in f32 for whole e in -126 .. 127, to the bit (pow on the GPU may be off by one in the last place)."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantized(v):
    """(values over their scales, exponents of the scales) of f32 v, in whole blocks: [rows, blocks, 32] and [rows, blocks]."""
    rows, n = v.shape
    pad = torch.zeros(rows, _blocks(n) * 32, device=v.device)
    pad[:, :n] = v
    blocks = pad.view(rows, -1, 32)
    e = torch.frexp(blocks.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -120))[1] - 3     # frexp's fraction is in [1/2, 1)
    a = (blocks / _power_of_two(e)).abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(((a / step).round() * step).clamp_max(6.0), blocks), e.squeeze(-1)


def _packed(v):
    """Codes [rows, 64 a group] and scale bytes [groups, rows padded to a multiple of four, 4] of f32 v, both uint8."""
    rows, n = v.shape
    q, e = _quantized(v)
    a = q.abs()
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8) + 8 * torch.signbit(q).to(torch.uint8)
    groups = -(-n // 128)
    codes = torch.zeros(rows, groups * 128, dtype=torch.uint8, device=v.device)
    codes[:, :code.shape[1] * 32] = code.view(rows, -1)
    exps = torch.full((-(-rows // 4) * 4, groups * 4), 127, dtype=torch.uint8, device=v.device)
    exps[:rows, :e.shape[1]] = (e + 127).to(torch.uint8)
    return codes[:, ::2] + 16 * codes[:, 1::2], exps.view(-1, groups, 4).transpose(0, 1).contiguous()


def _unpacked(codes, exps, n):
    """The values that codes stand for, f32 [rows, n]."""
    c = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1).to(torch.int32)
    m, top = (c & 1).float(), (c >> 1) & 3
    a = torch.where(top == 0, 0.5 * m, (1.0 + 0.5 * m) * _power_of_two(top - 1))
    e = exps.transpose(0, 1).reshape(exps.shape[1], -1)[:codes.shape[0]].to(torch.int32)
    v = torch.where(c >= 8, -a, a) * _power_of_two(e - 127).repeat_interleave(32, 1)
    return v[:, :n]


def _philox(key, counter):
    """Four words (int64 tensors that hold 32 bits) of ten rounds on the four words of `counter`."""
    low = 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    k0, k1 = key & low, key >> 32 & low
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57            # (wraps at 64 bits, all of which are wanted)
        c0, c1, c2, c3 = (p1 >> 32 & low) ^ c1 ^ k0, p1 & low, (p0 >> 32 & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _kept(rows, n, p, seed, offset):
    """(truth values [rows, n], the factor of what is kept)"""
    q = math.floor(65536 * p + 0.5)
    groups = -(-n // 8)
    row = torch.arange(rows, device="cuda").view(-1, 1).expand(rows, groups)
    group = torch.arange(groups, device="cuda").expand(rows, groups)
    words = _philox(seed, (group, row, torch.full_like(row, offset & 0xFFFFFFFF), torch.full_like(row, offset >> 32)))
    u = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], -1).view(rows, groups * 8)[:, :n]
    return u >= q, 65536.0 / (65536 - q)


def _normed(v, kind, w, b):
    """(norm, normalised v, r)"""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt(v.square().mean(-1, keepdim=True) + _EPS)
    v = v * r
    y = v if w is None else v * w
    return (y if b is None else y + b), v, r


def _normed_backward(g, kind, vh, r, w):
    """(gradient of v, of w, of b)"""
    t = g if w is None else g * w
    d = t - vh * (t * vh).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - t.mean(-1, keepdim=True)
    return r * d, (g * vh).sum(0), g.sum(0)


def _sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def _plain(s):
    case = s["case"]
    kind, t = case["kind"], _TYPES[case["dtype"]]
    if kind == "linear4":
        return {"y": _plain_linear(s, case).to(t)}
    shape = s["x"].shape
    rows, n = shape[0] * shape[1], shape[2]
    x = s["x"].detach().float().view(rows, n)
    if kind == "held4":
        q, e = _quantized(x)
        return {"x": (q * _power_of_two(e).unsqueeze(-1)).view(rows, -1)[:, :n].to(t).view(shape)}
    v = {k: s[k].detach().float() for k in ("w", "b", "nw", "nb", "scale") if s.get(k) is not None}
    if kind == "drop":
        kept, factor = _kept(rows, n, case["p"], s["seed"], s["offset"])
        out = {"y": torch.where(kept, x * factor, 0.0), "dx": torch.where(kept, s["gy"].float().view(rows, n) * factor, 0.0)}
    elif kind.startswith("norm"):
        h, xh, r = _normed(x, case["norm"], v["nw"], v.get("nb"))
        out = {"h": h}
        if kind == "norm_train":
            out["dx"], out["dnw"], out["dnb"] = _normed_backward(s["gh"].float().view(rows, n), case["norm"], xh, r, v["nw"])
            if s["nb"] is None:
                del out["dnb"]
    else:
        out = _plain_block(s, case, x, v, rows, n)
    return {k: o.to(t).view(shape) if k in ("y", "h", "dx", "df") else o.to(t) for k, o in out.items()}


def _plain_block(s, case, x, v, rows, n):
    f = s["f"].detach().float().view(rows, n)
    P, fh, fr = _normed(f, case["norm"], v.get("w"), v.get("b")) if case["norm"] != "none" else (f, f, None)
    u = torch.ones(1, n, device="cuda")
    act = slope = None
    if s["gate"] is not None:
        gate = s["gate"].detach().float().expand(s["x"].shape).reshape(rows, n)
        act, slope = gate, torch.ones_like(gate)
        if case["act"] == "sigmoid":
            act = _sigmoid(gate)
            slope = act * (1.0 - act)
        elif case["act"] == "silu":
            sg = _sigmoid(gate)
            act, slope = gate * sg, sg * (1.0 + gate * (1.0 - sg))
        u = act
    if "scale" in v:
        u = u * v["scale"]
    c = u * P
    kept = None
    if case["p"] > 0:
        kept, factor = _kept(rows, n, case["p"], s["seed"], s["offset"])
        c = torch.where(kept, c * factor, 0.0)
    y = x + c
    out = {"y": y}
    after = case["next_norm"] != "none"
    if after:
        out["h"], yh, yr = _normed(y, case["next_norm"], v["nw"], v.get("nb"))
    if case["kind"] == "block":
        return out
    d = s["gy"].float().view(rows, n)
    if after:
        more, out["dnw"], out["dnb"] = _normed_backward(s["gh"].float().view(rows, n), case["next_norm"], yh, yr, v["nw"])
        d = d + more
        if "nb" not in v:
            del out["dnb"]
    out["dx"] = d
    if kept is not None:
        d = torch.where(kept, d * factor, 0.0)
    if "scale" in v:
        out["dscale"] = (d * P if act is None else d * act * P).sum(0)
    if act is not None:
        dg = d * P * slope * (v["scale"] if "scale" in v else 1.0)
        dg = dg.view(s["x"].shape)
        out["dgate"] = dg.sum(1, keepdim=True) if case["gate"] == "sequence" else dg
    d = d * u
    if case["norm"] == "none":
        out["df"] = d
    else:
        out["df"], out["dw"], out["db"] = _normed_backward(d, case["norm"], fh, fr, v["w"])
        if "b" not in v:
            del out["db"]
    return out


def _plain_linear(s, case):
    q, e = _quantized(s["x"].float())
    x = (q * _power_of_two(e).unsqueeze(-1)).view(case["M"], -1)[:, :case["K"]]
    z = x @ _unpacked(s["w4"], s["we"], case["K"]).t()
    if s["b"] is not None:
        z = z + s["b"].float()
    if case["act"] == "relu":
        z = torch.where(z <= 0, 0.0, z)
    elif case["act"] == "gelu":
        z = 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    elif case["act"] == "silu":
        z = z * _sigmoid(z)
    return z if s["r"] is None else z + s["r"].float()


def _kernels(s):
    from paper_2204_03643_amd import block, quant4

    case = s["case"]
    kind = case["kind"]
    if kind == "linear4":
        w = quant4.Quantized4(s["w4"], s["we"], (case["N"], case["K"]), s["x"].dtype)
        return {"y": quant4.tv_linear4(s["x"], w, s["b"], s["r"], act=case["act"])}
    if kind == "held4":
        return {"x": quant4.tv_quantize4(s["x"]).restore()}
    if kind == "drop":
        y = block.tv_dropout(s["x"], case["p"], s["seed"], s["offset"])
        return {"y": y.detach(), "dx": torch.autograd.grad(y, s["x"], s["gy"])[0]}
    if kind.startswith("norm"):
        h = block.tv_norm(s["x"], s["nw"], s["nb"], kind=case["norm"], eps=_EPS)
        outs, gs = {"h": h}, [s.get("gh")]
    else:
        made = block.tv_residual(s["x"], s["f"], norm=case["norm"], weight=s["w"], bias=s["b"], gate=s["gate"],
                                 gate_act=case["act"], scale=s["scale"], dropout=case["p"], seed=s["seed"],
                                 offset=s["offset"], next_norm=case["next_norm"], next_weight=s["nw"],
                                 next_bias=s["nb"], eps=_EPS)
        outs = {"y": made} if case["next_norm"] == "none" else {"y": made[0], "h": made[1]}
        gs = [s.get("gy"), s.get("gh")][:len(outs)]
    if not kind.endswith("train"):
        return outs
    grads = torch.autograd.grad(list(outs.values()), [s[k] for k in s["leaves"]], gs)
    out = {k: o.detach() for k, o in outs.items()}
    out.update(("d" + k, g) for k, g in zip(s["leaves"], grads))
    return out


def run(state):
    out = _kernels(state) if own else _plain(state)
    return {k: out[k] for k in sorted(out)}


def work(case):
    size = {"f32": 4, "bf16": 2}[case["dtype"]]
    kind = case["kind"]
    if kind == "linear4":
        M, K, N = case["M"], case["K"], case["N"]
        values = M * K + M * N + (M * N if case["residual"] else 0) + (N if case["bias"] else 0)
        return {"bytes": size * values + N * (K // 2 + _blocks(K)), "flops": 2 * M * N * K}
    cells = case["B"] * case["T"] * case["n"]
    if kind == "held4":
        # in, the codes written and read, out
        return {"bytes": 2 * size * cells + 2 * case["T"] * (case["n"] // 2 + _blocks(case["n"])), "flops": 6 * cells}
    if kind == "drop":
        return {"bytes": 4 * size * cells, "flops": 2 * cells}
    # a training step reads again in its second half what it cannot keep on the chip; vectors of n are beside the point
    if kind.startswith("norm"):
        return {"bytes": size * cells * (5 if kind == "norm_train" else 2), "flops": cells * (16 if kind == "norm_train" else 6)}
    after, train = case["next_norm"] != "none", kind == "block_train"
    token, sequence = case["gate"] == "token", case["gate"] == "sequence"
    arrays = 3 + after + token                                # x, f, y; h; gate
    flops = 3 + 6 * (case["norm"] != "none") + 6 * after
    if train:
        arrays += 4 + 2 * after + 2 * token                   # dy, f, dx, df; dh, y; gate and its gradient
        flops *= 3
    rows = case["B"] * case["n"] * (2 if train else 1) if sequence else 0
    return {"bytes": size * (cells * arrays + rows), "flops": flops * cells}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]

    def wide(name):
        return s[name].detach().double() if s.get(name) is not None else None

    def in_four_bits(v):
        """By comparison with the seven borders between neighbouring values, a block of columns at a time."""
        values = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=v.device)
        out = torch.empty_like(v)
        for first in range(0, v.shape[-1], 32):
            part = v[..., first:first + 32]
            top = torch.clamp(part.abs().max(dim=-1, keepdim=True).values, min=2.0 ** -120)
            scale = torch.exp2(torch.floor(torch.log2(top)) - 2)
            # log2 may round across a power of two; the scale itself is made exact by its exponent field
            scale = (((torch.log2(scale).round().long() + 1023) << 52).view(torch.float64))
            scale = torch.where(top / scale >= 8, scale * 2, torch.where(top / scale < 4, scale / 2, scale))
            a = part.abs() / scale
            at = torch.zeros_like(a, dtype=torch.long)
            for border, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
                at += (a >= border) if up else (a > border)
            out[..., first:first + 32] = values[at] * scale * torch.where(part < 0, -1.0, 1.0)
        return out

    def dropped(rows, n, p):
        """True where a channel is dropped: the generator's products by halves of 16 bits."""
        def both(c, m):
            lo, hi, ml, mh = c & 0xFFFF, c >> 16, m & 0xFFFF, m >> 16
            mid = hi * ml + (lo * ml >> 16)                   # below 2^33
            mid2 = lo * mh + (mid & 0xFFFF)
            return hi * mh + (mid >> 16) + (mid2 >> 16), (mid2 & 0xFFFF) << 16 | (lo * ml & 0xFFFF)
        at = torch.cartesian_prod(torch.arange(rows, device="cuda"), torch.arange((n + 7) // 8, device="cuda")).view(-1, 2)
        word = [at[:, 1], at[:, 0], torch.zeros_like(at[:, 0]) + s["offset"] % 2 ** 32, torch.zeros_like(at[:, 0]) + s["offset"] // 2 ** 32]
        for turn in range(10):
            keys = [(s["seed"] % 2 ** 32 + turn * 0x9E3779B9) % 2 ** 32, (s["seed"] // 2 ** 32 + turn * 0xBB67AE85) % 2 ** 32]
            h0, l0 = both(word[0], 0xD2511F53)
            h1, l1 = both(word[2], 0xCD9E8D57)
            word = [h1 ^ word[1] ^ keys[0], l1, h0 ^ word[3] ^ keys[1], l0]
        u = torch.empty(len(at), 8, dtype=torch.long, device="cuda")
        for i in range(8):
            u[:, i] = torch.div(word[i // 2], 65536, rounding_mode="floor") if i % 2 else torch.remainder(word[i // 2], 65536)
        return u.view(rows, -1)[:, :n] < int(65536 * p + 0.5)

    if kind == "linear4":
        w = torch.zeros(case["N"], s["w4"].shape[1] * 2, dtype=torch.float64, device="cuda")
        stands = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device="cuda")
        w[:, 0::2] = stands[torch.remainder(s["w4"].long(), 16)]
        w[:, 1::2] = stands[torch.div(s["w4"].long(), 16, rounding_mode="floor")]
        scales = ((s["we"].long() - 127 + 1023) << 52).view(torch.float64)
        for group in range(scales.shape[0]):
            for i in range(4):
                first = group * 128 + i * 32
                w[:, first:first + 32] *= scales[group, :case["N"], i].unsqueeze(1)
        w = w[:, :case["K"]]
        y = torch.matmul(in_four_bits(wide("x")), w.transpose(0, 1).contiguous())
        if s["b"] is not None:
            y += wide("b")
        if case["act"] == "relu":
            y = torch.clamp(y, min=0)
        elif case["act"] == "gelu":
            y = y * torch.special.erfc(-y / math.sqrt(2.0)) / 2
        elif case["act"] == "silu":
            y = y * torch.sigmoid(y)
        if s["r"] is not None:
            y += wide("r")
        return {"y": y}
    x = wide("x")
    B, T, n = x.shape
    if kind == "held4":
        return {"x": in_four_bits(x)}
    if kind == "drop":
        gone = dropped(B * T, n, case["p"]).view(B, T, n)
        keep = 1.0 - int(65536 * case["p"] + 0.5) / 65536.0
        return {"dx": (wide("gy") / keep).masked_fill(gone, 0.0), "y": (x / keep).masked_fill(gone, 0.0)}

    def unit(v, layer):
        m = v.mean(dim=-1, keepdim=True) if layer else 0.0
        std = ((v - m).pow(2).sum(dim=-1, keepdim=True) / n + _EPS).sqrt()
        return (v - m) / std, std

    def unit_gradient(t, vh, std, layer):
        out = t - vh * (t * vh).sum(dim=-1, keepdim=True) / n
        if layer:
            out = out - t.sum(dim=-1, keepdim=True) / n
        return out / std

    def over_rows(v):
        return v.sum(dim=(0, 1))

    out = {}
    if kind.startswith("norm"):
        layer = case["norm"] == "layer"
        xh, std = unit(x, layer)
        out["h"] = xh * wide("nw") + (wide("nb") if case["bias"] else 0.0)
        if kind == "norm_train":
            g = wide("gh")
            out["dx"] = unit_gradient(g * wide("nw"), xh, std, layer)
            out["dnw"] = over_rows(g * xh)
            if case["bias"]:
                out["dnb"] = over_rows(g)
        return {k: out[k] for k in sorted(out)}
    f, layer = wide("f"), case["norm"] == "layer"
    fh, fstd = unit(f, layer) if case["norm"] != "none" else (f, None)
    P = fh
    if s["w"] is not None:
        P = P * wide("w")
    if s["b"] is not None:
        P = P + wide("b")
    scale = wide("scale") if s["scale"] is not None else torch.ones(n, dtype=torch.float64, device="cuda")
    G, dG = 1.0, None
    if s["gate"] is not None:
        z = wide("gate")
        G, dG = z, torch.ones_like(z)
        if case["act"] != "none":
            sg, other = torch.sigmoid(z), torch.sigmoid(-z)
            G, dG = (sg, sg * other) if case["act"] == "sigmoid" else (z * sg, sg + z * sg * other)
    d = torch.ones_like(x)
    if case["p"] > 0:
        d = (d / (1.0 - int(65536 * case["p"] + 0.5) / 65536.0)).masked_fill(dropped(B * T, n, case["p"]).view(B, T, n), 0.0)
    y = x + d * scale * G * P
    out["y"] = y
    if case["next_norm"] != "none":
        yh, ystd = unit(y, case["next_norm"] == "layer")
        out["h"] = yh * wide("nw") + (wide("nb") if s["nb"] is not None else 0.0)
    if kind == "block_train":
        dy = wide("gy")
        if case["next_norm"] != "none":
            gh = wide("gh")
            dy = dy + unit_gradient(gh * wide("nw"), yh, ystd, case["next_norm"] == "layer")
            out["dnw"] = over_rows(gh * yh)
            if s["nb"] is not None:
                out["dnb"] = over_rows(gh)
        out["dx"] = dy
        dc = dy * d
        if s["scale"] is not None:
            out["dscale"] = over_rows(dc * G * P)
        if dG is not None:
            dgate = dc * scale * P * dG
            out["dgate"] = dgate.sum(dim=1, keepdim=True) if case["gate"] == "sequence" else dgate
        dP = dc * scale * G
        if case["norm"] == "none":
            out["df"] = dP
        else:
            out["dw"] = over_rows(dP * fh)
            if s["b"] is not None:
                out["db"] = over_rows(dP)
            out["df"] = unit_gradient(dP * wide("w"), fh, fstd, layer)
    return {k: out[k] for k in sorted(out)}
