// C-ABI entry points of the channel products and the 8-bit checkpoints: argument validation, choice of kernels,
// workspace layout and launches.
#include "../../include/tvprox.h"
#include "tv_ckpt8.hpp"
#include "tv_gemm_split.hpp"
#include "tv_gemv.hpp"
#include "tv_slope.hpp"

namespace {

using namespace tvl;

constexpr int64_t kMostIndex = (int64_t)1 << 31;      // sizes and strides stay below
constexpr int64_t kMostTiles = (int64_t)1 << 22;      // workgroups of a launch

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t tiles(int64_t v, int64_t of) { return (v + of - 1) / of; }
size_t elem_bytes(int dtype) { return dtype == TV_BF16 ? 2 : 4; }
bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }
int launched() { return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP; }

// ---- products
// One operand: rows of `cols` elements, ld apart; padded: readable, and zero, up to a multiple of eight columns.
struct Operand {
    const void *p;
    int64_t ld, cols;
    bool padded;
};

constexpr int64_t kFewRows = 64;

// Which kernel a product takes and how its contraction is split, from sizes and alignment alone.
enum Kind { kFew, kTile256, kTile128, kTile128Deep, kTile64, kSplit256, kSplit128, kSplit64 };
struct Choice {
    Kind kind;
    int splits, k_per;
};

struct Tile { int m, n; };
Tile tile_of_kind(Kind k)
{
    if (k == kTile256 || k == kSplit256) return {256, 256};
    if (k == kTile64 || k == kSplit64) return {64, 128};
    return {128, 128};
}

int64_t few_columns(int64_t) { return 32; }

// `s` splits of a contraction of K, each a multiple of `unit`
Choice cut(Kind kind, int64_t s, int64_t K, int64_t unit)
{
    if (s < 1) s = 1;
    const int64_t per = up(K > 0 ? tiles(K, s) : 1, unit);
    return {kind, (int)(K > 0 ? tiles(K, per) : 1), (int)per};
}

Choice choose(int dtype, bool direct, bool transposed, int64_t M, int64_t N, int64_t K)
{
    if (!transposed && M >= 1 && M <= (direct && dtype == TV_BF16 ? kFewRows / 2 : kFewRows)) {
        const int64_t turn = 8 * 64 / (int64_t)elem_bytes(dtype);            // a turn of all eight waves
        const int64_t t = tiles(N, few_columns(M));
        const int64_t s = t >= 256 ? 1 : 256 / t;
        return cut(kFew, s < K / (8 * turn) ? s : K / (8 * turn), K, turn);
    }
    /*SWEEP*/
    // The cheapest by a model of the time in microseconds, fitted to sweeps of tiles and splits over outputs of
    // 128 x 128 to 8192 x 8192 and contractions of 64 to 8192: a launch, rounds of workgroups over 256 compute units (of
    // two workgroups each where there are more than 256 of a kernel that leaves room for two), in each a start and an end
    // and so much a step of 64, and for split contractions the second launch and the sums' trip through memory.
    struct Cost { Kind kind; int64_t slots; double round, step; };
    constexpr Cost direct16[] = {{kTile64, 256, 1.0, 0.30}, {kTile128Deep, 256, 2.0, 0.47}, {kTile128, 512, 3.0, 0.88}, {kTile256, 256, 6.5, 1.50}};
    constexpr Cost any16[] = {{kSplit64, 256, 1.5, 0.62}, {kSplit64, 512, 2.0, 0.85}, {kSplit128, 256, 3.0, 0.95}};
    constexpr Cost any32[] = {{kSplit64, 256, 2.5, 1.35}, {kSplit128, 256, 3.5, 2.65}, {kSplit256, 256, 8.0, 9.0}};
    const Cost *costs = dtype != TV_BF16 ? any32 : direct ? direct16 : any16;
    const int kinds = dtype == TV_BF16 && direct ? 4 : 3;
    Choice best = cut(costs[0].kind, 1, K, 64);
    double least = 1e30;
    for (int i = 0; i < kinds; ++i) {
        const Cost &c = costs[i];
        const Tile side = tile_of_kind(c.kind);
        const int64_t t = tiles(M, side.m) * tiles(N, side.n);
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (s > 1 && (K < 128 * s || t * s > 1024)) break;
            const Choice x = cut(c.kind, s, K, 64);
            double us = 3.0 + (double)tiles(t * x.splits, c.slots) * (c.round + c.step * (double)tiles(x.k_per < K ? x.k_per : K, 64));
            if (x.splits > 1) us += 4.0 + (double)M * (double)N * x.splits * 8 / 6e6;
            if (us < least) { least = us; best = x; }
        }
    }
    return best;
}

size_t split_bytes(const Choice &c, int64_t M, int64_t N)
{
    return c.splits > 1 ? (size_t)up((int64_t)c.splits * M * up(N, 8) * 4, 256) : 0;
}

bool product_fits(int64_t M, int64_t N) { return tiles(M, 128) * tiles(N, 128) <= kMostTiles; }

// Rows on 16-byte boundaries, whole 16-byte pieces, and offsets within a tile of 256 rows that 32 bits hold.
bool direct(const Operand &o)
{
    return aligned(o.p, 16) && o.ld % 8 == 0 && (o.cols % 8 == 0 || o.padded) && o.ld <= ((int64_t)1 << 22);
}

template <int BM, int BN, int THREADS>
void launch_tiles(void (*kernel)(Product, Epilogue), Product g, const Epilogue &e, hipStream_t stream)
{
    g.tiles_m = (uint32_t)tiles(g.M, BM);
    g.tiles_n = (uint32_t)tiles(g.N, BN);
    hipLaunchKernelGGL(kernel, dim3(g.tiles_m * g.tiles_n, g.splits), dim3(THREADS), 0, stream, g, e);
}

template <class T, class TB, bool AT, bool BT>
int run_product(const Operand &a, const Operand &b, int64_t M, int64_t N, int64_t K, const Choice &c, const Epilogue &e,
                void *ws, hipStream_t stream)
{
    Product g{a.p, b.p, a.ld, b.ld, (int32_t)M, (int32_t)N, (int32_t)K, c.k_per, c.splits, (float *)ws, 0, 0};
    if constexpr (sizeof(T) == 2) {
        if (c.kind == kTile256) launch_tiles<256, 256, 512>(gemm16_kernel<256, 256, 2, 4, 2, AT, BT>, g, e, stream);
        if (c.kind == kTile128) launch_tiles<128, 128, 256>(gemm16_kernel<128, 128, 2, 2, 2, AT, BT>, g, e, stream);
        if (c.kind == kTile128Deep) launch_tiles<128, 128, 256>(gemm16_kernel<128, 128, 2, 2, 4, AT, BT>, g, e, stream);
        if (c.kind == kTile64) launch_tiles<64, 128, 256>(gemm16_kernel<64, 128, 2, 2, 4, AT, BT>, g, e, stream);
        if (c.kind == kSplit128) launch_tiles<128, 128, 256>(gemm_split_kernel<T, TB, 128, 128, 2, 2, 4, 2, 1, AT, BT>, g, e, stream);
        if (c.kind == kSplit64) launch_tiles<64, 128, 256>(gemm_split_kernel<T, TB, 64, 128, 2, 2, 4, 2, 1, AT, BT>, g, e, stream);
    } else {
        if (c.kind == kSplit256) launch_tiles<256, 256, 512>(gemm_split_kernel<T, TB, 256, 256, 2, 4, 1, 1, 1, AT, BT>, g, e, stream);
        if (c.kind == kSplit128) launch_tiles<128, 128, 512>(gemm_split_kernel<T, TB, 128, 128, 4, 2, 2, 2, 1, AT, BT>, g, e, stream);
        if (c.kind == kSplit64) launch_tiles<64, 128, 512>(gemm_split_kernel<T, TB, 64, 128, 2, 2, 4, 2, 2, AT, BT>, g, e, stream);
    }
    if constexpr (!AT && !BT)
        if (c.kind == kFew) {
            const dim3 grid((uint32_t)tiles(N, few_columns(M)), c.splits), block(512);
            if (M <= 16) hipLaunchKernelGGL((gemv_kernel<T, 1, 2, 8>), grid, block, 0, stream, g, e);
            else if (M <= 32) hipLaunchKernelGGL((gemv_kernel<T, 2, 2, 8>), grid, block, 0, stream, g, e);
            else hipLaunchKernelGGL((gemv_kernel<T, 4, 2, 4>), grid, block, 0, stream, g, e);
        }
    if (c.splits > 1) {
        if (launched() != TV_OK) return TV_ERR_HIP;
        hipLaunchKernelGGL((join_kernel<T>), dim3((uint32_t)tiles(M * tiles(N, 32) * 4, 256)), dim3(256), 0, stream, g, e);
    }
    return launched();
}

Epilogue plain_output(void *y, int64_t ldy)
{
    Epilogue e{};
    e.y = y; e.ldy = ldy;
    return e;
}

// ---- validation
int check_sizes(const tv_linear_desc &d)
{
    if (d.m < 0 || d.k < 1 || d.n < 1 || d.m >= kMostIndex || d.k >= kMostIndex - 128 || d.n >= kMostIndex - 128) return TV_ERR_SHAPE;
    if (!product_fits(d.m, d.n) || !product_fits(d.m, d.k) || !product_fits(d.n, d.k)) return TV_ERR_SHAPE;
    if ((d.dtype != TV_F32 && d.dtype != TV_BF16) || d.act < TV_ACT_NONE || d.act > TV_ACT_SILU) return TV_ERR_UNSUPPORTED;
    if (d.ldx < d.k || d.ldw < d.k || d.ldy < d.n || d.ldx >= kMostIndex || d.ldw >= kMostIndex || d.ldy >= kMostIndex) return TV_ERR_STRIDE;
    return TV_OK;
}

int check_held(const tv_linear_desc &d, const tv_held &h, bool needed)
{
    const bool smooth = d.act == TV_ACT_GELU || d.act == TV_ACT_SILU;
    switch (h.kind) {
    case TV_HELD_NONE: return needed && d.act != TV_ACT_NONE ? TV_ERR_UNSUPPORTED : TV_OK;
    case TV_HELD_BITS:
        if (d.act != TV_ACT_RELU) return TV_ERR_UNSUPPORTED;
        break;
    case TV_HELD_PLAIN:
    case TV_HELD_8BIT:
        if (!smooth) return TV_ERR_UNSUPPORTED;
        break;
    default: return TV_ERR_UNSUPPORTED;
    }
    if (d.m == 0) return TV_OK;
    if (!h.data || (h.kind == TV_HELD_8BIT && !h.exps)) return TV_ERR_NULL;
    const size_t to = h.kind == TV_HELD_BITS ? 4 : h.kind == TV_HELD_PLAIN ? elem_bytes(d.dtype) : 1;
    return aligned(h.data, to) ? TV_OK : TV_ERR_STRIDE;
}

int check_workspace(const void *ws, size_t have, size_t need)
{
    return need && (!ws || !aligned(ws, 16) || have < need) ? TV_ERR_WORKSPACE : TV_OK;
}

Choice fwd_choice(const tv_linear_desc &d, const void *x, const void *w)
{
    return choose(d.dtype, direct({x, d.ldx, d.k, false}) && direct({w, d.ldw, d.k, false}), false, d.m, d.n, d.k);
}

// (The workspace is asked for before there are pointers, and has to do for either choice.)
size_t fwd_bytes(const tv_linear_desc &d)
{
    const size_t a = split_bytes(choose(d.dtype, true, false, d.m, d.n, d.k), d.m, d.n);
    const size_t b = split_bytes(choose(d.dtype, false, false, d.m, d.n, d.k), d.m, d.n);
    return a > b ? a : b;
}

template <class T>
int linear_fwd(const void *x, const void *w, const void *bias, const void *res, void *y, const tv_held &h,
               const tv_linear_desc &d, const Choice &c, void *ws, hipStream_t stream)
{
    Epilogue e{};
    e.bias = bias; e.res = res; e.y = y;
    e.held = h.kind == TV_HELD_NONE ? nullptr : h.data; e.exps = h.exps;
    e.ldr = d.ldr; e.ldy = d.ldy; e.act = d.act; e.kind = h.kind;
    return run_product<T, T, false, false>({x, d.ldx, d.k, false}, {w, d.ldw, d.k, false}, d.m, d.n, d.k, c, e, ws, stream);
}

// ---- the backward call's workspace: dz, x out of its checkpoint, the column sums of groups of rows, split sums
struct BwdPlan {
    size_t dz, x, sums, split, bytes;
    int64_t ldz, ldx;
    int rows_per, groups;
};

BwdPlan bwd_plan(const tv_linear_desc &d, bool x8)
{
    BwdPlan p{};
    const size_t size = elem_bytes(d.dtype);
    size_t at = 0;
    p.ldz = up(d.n, 8);
    p.dz = at;
    if (d.act != TV_ACT_NONE) at += up(d.m * p.ldz * (int64_t)size, 256);
    p.ldx = up(d.k, 8);
    p.x = at;
    if (x8) at += up(d.m * p.ldx * 2, 256);
    // about 1024 workgroups of 256 columns each, of sixteen rows at least
    const int64_t want = 1024 / tiles(d.n, 256) + 1;
    p.rows_per = (int)(d.m > 64 ? up(tiles(d.m, want < 256 ? want : 256), 16) : 64);       // (up to 64 rows: one group, one launch)
    p.groups = (int)tiles(d.m, p.rows_per);
    p.sums = at;
    at += up((int64_t)p.groups * d.n * 4, 256);
    p.split = at;
    size_t most = 0;
    for (bool dir : {false, true}) {
        const size_t s1 = split_bytes(choose(d.dtype, dir, true, d.m, d.k, d.n), d.m, d.k);
        const size_t s2 = split_bytes(choose(d.dtype, dir, true, d.n, d.k, d.m), d.n, d.k);
        most = most > s1 ? most : s1;
        most = most > s2 ? most : s2;
    }
    p.bytes = at + most;
    return p;
}

template <class T>
int linear_bwd(const void *g, const void *x, const uint8_t *x_exps, const tv_held &h, const void *w, void *dx, void *dw,
               void *db, const tv_linear_desc &d, char *ws, hipStream_t stream)
{
    const BwdPlan p = bwd_plan(d, x_exps != nullptr);
    Operand dz{g, d.ldy, d.n, false};
    if (d.m > 0 && (d.act != TV_ACT_NONE || db)) {
        SlopeArgs a{};
        a.g = g; a.held = h.data; a.exps = h.exps;
        a.dz = d.act != TV_ACT_NONE ? ws + p.dz : nullptr;
        a.sums = db && p.groups > 1 ? (float *)(ws + p.sums) : nullptr;
        a.db = p.groups == 1 ? db : nullptr;
        a.ldg = d.ldy; a.ldz = p.ldz;
        a.M = (int32_t)d.m; a.N = (int32_t)d.n; a.rows_per = p.rows_per;
        a.act = d.act; a.kind = d.act == TV_ACT_NONE ? TV_HELD_NONE : h.kind;
        hipLaunchKernelGGL((slope_kernel<T>), dim3((uint32_t)tiles(d.n, 256), p.groups), dim3(256), 0, stream, a);
        if (launched() != TV_OK) return TV_ERR_HIP;
        if (a.dz) dz = {a.dz, p.ldz, d.n, false};
    }
    if (db && p.groups != 1) {
        hipLaunchKernelGGL((column_sum_kernel<T>), dim3((uint32_t)tiles(d.n, 32)), dim3(256), 0, stream,
                           (const float *)(ws + p.sums), (T *)db, d.m > 0 ? p.groups : 0, (int)d.n);
        if (launched() != TV_OK) return TV_ERR_HIP;
    }
    if (dx && d.m > 0) {
        const Operand ow{w, d.ldw, d.k, false};
        const int st = run_product<T, T, false, true>(dz, ow, d.m, d.k, d.n, choose(d.dtype, direct(dz) && direct(ow), true, d.m, d.k, d.n),
                                                   plain_output(dx, d.k), ws + p.split, stream);
        if (st != TV_OK) return st;
    }
    if (dw) {
        Operand xs{x, d.ldx, d.k, false};
        if (x_exps && d.m > 0) {                      // what codes stand for is exact in bf16
            const int st = tv_ckpt8_load((const int8_t *)x, x_exps, ws + p.x, d.m, d.k, p.ldx, TV_BF16, stream);
            if (st != TV_OK) return st;
            xs = {ws + p.x, p.ldx, d.k, false};
        }
        const Choice c = choose(d.dtype, direct(dz) && direct(xs), true, d.n, d.k, d.m);
        const Epilogue e = plain_output(dw, d.k);
        return x_exps ? run_product<T, bf16, true, true>(dz, xs, d.n, d.k, d.m, c, e, ws + p.split, stream)
                      : run_product<T, T, true, true>(dz, xs, d.n, d.k, d.m, c, e, ws + p.split, stream);
    }
    return TV_OK;
}

int check_ckpt8(int64_t rows, int64_t n, int64_t ld, int dtype)
{
    if (rows < 0 || n < 1 || rows >= kMostIndex || n >= kMostIndex - 128) return TV_ERR_SHAPE;
    if (rows > ((int64_t)1 << 40) / n) return TV_ERR_SHAPE;
    if (dtype != TV_F32 && dtype != TV_BF16) return TV_ERR_UNSUPPORTED;
    if (ld < n || ld >= kMostIndex) return TV_ERR_STRIDE;
    return TV_OK;
}

dim3 ckpt8_grid(int64_t rows, int64_t n)
{
    const int64_t groups = tiles(rows * tiles(n, kBlock), 64), wide = (int64_t)1 << 22;
    return groups <= wide ? dim3((uint32_t)groups) : dim3((uint32_t)wide, (uint32_t)tiles(groups, wide));
}

}  // namespace

extern "C" {

size_t tv_linear_fwd_workspace_bytes(tv_linear_desc d)
{
    return check_sizes(d) == TV_OK ? fwd_bytes(d) : 0;
}

int tv_linear_fwd(const void *x, const void *w, const void *bias, const void *res, void *y, tv_held held,
                  tv_linear_desc d, void *ws, size_t ws_bytes, hipStream_t stream)
{
    int st = check_sizes(d);
    if (st != TV_OK) return st;
    if (res && (d.ldr < d.n || d.ldr >= kMostIndex)) return TV_ERR_STRIDE;
    if ((st = check_held(d, held, false)) != TV_OK) return st;
    if (d.m == 0) return TV_OK;
    if (!x || !w || !y) return TV_ERR_NULL;
    const size_t size = elem_bytes(d.dtype);
    if (!aligned(x, size) || !aligned(w, size) || !aligned(bias, size) || !aligned(res, size) || !aligned(y, size)) return TV_ERR_STRIDE;
    const Choice c = fwd_choice(d, x, w);
    if (c.splits > 1 && (st = check_workspace(ws, ws_bytes, fwd_bytes(d))) != TV_OK) return st;
    return d.dtype == TV_BF16 ? linear_fwd<bf16>(x, w, bias, res, y, held, d, c, ws, stream)
                              : linear_fwd<float>(x, w, bias, res, y, held, d, c, ws, stream);
}

size_t tv_linear_bwd_workspace_bytes(tv_linear_desc d, int x_is_8bit)
{
    return check_sizes(d) == TV_OK ? bwd_plan(d, x_is_8bit != 0).bytes : 0;
}

int tv_linear_bwd(const void *g, const void *x, const uint8_t *x_exps, tv_held held, const void *w, void *dx, void *dw,
                  void *db, tv_linear_desc d, void *ws, size_t ws_bytes, hipStream_t stream)
{
    int st = check_sizes(d);
    if (st != TV_OK) return st;
    if ((st = check_held(d, held, true)) != TV_OK) return st;
    if ((d.m > 0 && (!g || (dx && !w) || (dw && !x)))) return TV_ERR_NULL;
    const size_t size = elem_bytes(d.dtype);
    if (!aligned(g, size) || (!x_exps && !aligned(x, size)) || !aligned(w, size) || !aligned(dx, size) || !aligned(dw, size) ||
        !aligned(db, size)) return TV_ERR_STRIDE;
    if ((st = check_workspace(ws, ws_bytes, bwd_plan(d, x_exps != nullptr).bytes)) != TV_OK) return st;
    return d.dtype == TV_BF16 ? linear_bwd<bf16>(g, x, x_exps, held, w, dx, dw, db, d, (char *)ws, stream)
                              : linear_bwd<float>(g, x, x_exps, held, w, dx, dw, db, d, (char *)ws, stream);
}

int tv_ckpt8_save(const void *x, int8_t *codes, uint8_t *exps, int64_t rows, int64_t n, int64_t ldx, int dtype, hipStream_t stream)
{
    const int st = check_ckpt8(rows, n, ldx, dtype);
    if (st != TV_OK || rows == 0) return st;
    if (!x || !codes || !exps) return TV_ERR_NULL;
    const size_t size = elem_bytes(dtype);
    if (!aligned(x, size)) return TV_ERR_STRIDE;
    const int blocks = (int)tiles(n, kBlock);
    if (dtype == TV_BF16)
        hipLaunchKernelGGL((ckpt8_save_kernel<bf16>), ckpt8_grid(rows, n), dim3(256), 0, stream, (const bf16 *)x, ldx, codes, exps, rows, (int)n, blocks);
    else
        hipLaunchKernelGGL((ckpt8_save_kernel<float>), ckpt8_grid(rows, n), dim3(256), 0, stream, (const float *)x, ldx, codes, exps, rows, (int)n, blocks);
    return launched();
}

int tv_ckpt8_load(const int8_t *codes, const uint8_t *exps, void *x, int64_t rows, int64_t n, int64_t ldx, int dtype, hipStream_t stream)
{
    const int st = check_ckpt8(rows, n, ldx, dtype);
    if (st != TV_OK || rows == 0) return st;
    if (!x || !codes || !exps) return TV_ERR_NULL;
    const size_t size = elem_bytes(dtype);
    if (!aligned(x, size)) return TV_ERR_STRIDE;
    const int blocks = (int)tiles(n, kBlock);
    if (dtype == TV_BF16)
        hipLaunchKernelGGL((ckpt8_load_kernel<bf16>), ckpt8_grid(rows, n), dim3(256), 0, stream, codes, exps, (bf16 *)x, ldx, rows, (int)n, blocks);
    else
        hipLaunchKernelGGL((ckpt8_load_kernel<float>), ckpt8_grid(rows, n), dim3(256), 0, stream, codes, exps, (float *)x, ldx, rows, (int)n, blocks);
    return launched();
}

}  // extern "C"
