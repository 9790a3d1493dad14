// C-ABI entry points of the channel products and the 8-bit checkpoints: argument validation, choice of kernels,
// workspace layout and launches.
#include "../../include/tvprox.h"
#include "tv_ckpt8.hpp"
#include "tv_gemm_split.hpp"
#include "tv_gemv.hpp"
#include "tv_slope.hpp"

namespace {

using namespace tvl;

constexpr int64_t kMostIndex = ((int64_t)1 << 31) - 1024;      // sizes stay below: a step past the end fits 32 bits too
constexpr int64_t kMostStride = (int64_t)1 << 31;              // strides stay below
constexpr int64_t kMostTiles = TV_LINEAR_MAX_TILES;            // so that every launch has fewer than 2^32 threads

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t tiles(int64_t v, int64_t of) { return (v + of - 1) / of; }
size_t elem_bytes(int dtype) { return dtype == TV_BF16 ? 2 : 4; }
bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }
int launched() { return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP; }

// ---- products
// One operand: `rows` rows of `cols` elements, ld apart.
struct Operand {
    const void *p;
    int64_t ld, rows, cols;
};

// Rows on 16-byte boundaries, whole 16-byte pieces, and offsets within a tile of 256 rows that 32 bits hold.
bool direct(const Operand &o)
{
    return aligned(o.p, 16) && o.ld % 8 == 0 && o.cols % 8 == 0 && o.ld <= ((int64_t)1 << 22);
}

constexpr int64_t kFewRows = 64;

// Which kernel a product takes and how its contraction is split.
enum Kind { kFew, kTile256, kTile128, kTile128Deep, kTile64, kSplit256, kSplit128, kSplit64 };
struct Choice {
    Kind kind;
    int splits, k_per;
    double us;           // what the model says
};

struct Tile { int m, n; };
Tile tile_of_kind(Kind k)
{
    if (k == kTile256 || k == kSplit256) return {256, 256};
    if (k == kTile64 || k == kSplit64) return {64, 128};
    return {128, 128};
}

// `s` splits of a contraction of K, each a multiple of `unit`
Choice cut(Kind kind, int64_t s, int64_t K, int64_t unit)
{
    if (s < 1) s = 1;
    const int64_t per = up(K > 0 ? tiles(K, s) : 1, unit);
    return {kind, (int)(K > 0 ? tiles(K, per) : 1), (int)per, 0.0};
}

// Sizes, type and alignment alone decide.  Few rows stream the weight, where that is faster than tiles.  bf16 operands that
// go straight to LDS: up to 32 rows (2048 -> 8192, streamed and through tiles: 32 rows 11.6 and 12.8 us, 48 rows 14.7 and
// 13.8); f32 ones up to 16 (16 rows 22.7 and 23.2 us, 32 rows 28.4 and 23.8).  More rows, and rows on other boundaries, cost
// so much a turn of the waves that only short streams pay: turns one after the other, times the 2, 3 or 6 that one costs
// with up to 16, 32 or 64 rows, up to 36 in f32 (1024 -> 1024: 32 rows, 24, 9.1 and 12.2 us; 64 rows, 48,
// 14.1 and 12.8) and 12 in bf16 (1001 -> 777, 32 rows, 12: 9.0 and 10.8 us; 2047 -> 513, 16 rows, 16: 15.1 and 11.3).
//
// Otherwise the cheapest by a model of the time in microseconds, fitted to sweeps of tiles and splits over outputs of
// 128 x 512 to 8192 x 8192 and contractions of 256 to 16384 (what it takes there is 0.1 to 0.7 % slower than the best of the sweep, 11 %
// at most): a launch; rounds of workgroups over 256 compute units, in each a start and an end and so much a step of 64,
// more where two workgroups share a unit or, at lower clocks, where more than half of the units are busy; for split
// contractions the second launch and the sums' trip through memory.
struct Cost {
    Kind kind;
    int64_t slots;               // workgroups at a time
    double round, step, more;
};

double rounds_us(const Cost &c, int64_t workgroups, int64_t steps)
{
    const int64_t full = workgroups / c.slots, rest = workgroups % c.slots;
    // (the second half of 256 workgroups does not spread evenly where units take two)
    const double half = rest > 128 ? rest / 128.0 - 1.0 : 0.0, load = c.slots == 256 ? half : rest > 256 ? 1.0 : 0.5 * half;
    double us = (double)full * (c.round + (c.step + c.more) * (double)steps);
    if (rest) us += c.round + (c.step + c.more * load) * (double)steps;
    return us;
}

Choice choose(int dtype, bool direct, bool transposed, int64_t M, int64_t N, int64_t K)
{
    if (!transposed && M >= 1 && M <= kFewRows) {
        const int64_t turn = 8 * 64 / (int64_t)elem_bytes(dtype);            // a turn of all eight waves
        const int64_t t = tiles(N, 32), s = t >= 256 ? 1 : 256 / t;
        const Choice x = cut(kFew, s < K / (8 * turn) ? s : K / (8 * turn), K, turn);
        const int64_t turns = tiles(t * x.splits, 256) * tiles(x.k_per < K ? x.k_per : K, turn);
        if ((direct && M <= (dtype == TV_BF16 ? 32 : 16)) || turns * (M <= 16 ? 2 : M <= 32 ? 3 : 6) <= (dtype == TV_BF16 ? 12 : 36)) return x;
    }
    constexpr Cost direct16[] = {{kTile64, 256, 1.0, 0.25, 0.08}, {kTile128Deep, 256, 1.8, 0.38, 0.13}, {kTile128, 512, 1.5, 0.42, 0.52}, {kTile256, 256, 4.2, 1.14, 0.49}};
    constexpr Cost any16[] = {{kSplit64, 512, 3.2, 0.45, 0.44}};
    constexpr Cost any32[] = {{kSplit64, 256, 4.2, 1.26, 0.35}, {kSplit128, 256, 3.6, 1.97, 0.80}, {kSplit256, 256, 7.4, 6.6, 2.5}};
    const Cost *costs = dtype != TV_BF16 ? any32 : direct ? direct16 : any16;
    const int kinds = dtype != TV_BF16 ? 3 : direct ? 4 : 1;
    Choice best = cut(costs[0].kind, 1, K, 64);
    best.us = 1e30;
    for (int i = 0; i < kinds; ++i) {
        const Cost &c = costs[i];
        const Tile side = tile_of_kind(c.kind);
        const int64_t t = tiles(M, side.m) * tiles(N, side.n);
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (s > 1 && (K < 128 * s || t * s > 1024)) break;
            Choice x = cut(c.kind, s, K, 64);
            x.us = 3.0 + rounds_us(c, t * x.splits, tiles(x.k_per < K ? x.k_per : K, 64));
            if (x.splits > 1) x.us += 2.6 + 0.18 * x.splits + (double)M * (double)N * x.splits * 8 / 7e6;
            if (x.us < best.us) best = x;
        }
    }
    return best;
}

// bf16 operands that cannot go straight to LDS are copied to rows that can, where the faster kernel pays for it
// (8192 x 2047 -> 8191: 505 us without, 250 with): a launch and the bytes there and back each.
struct Plan {
    Choice c;
    bool copy_a, copy_b;
};
double copy_us(int64_t rows, int64_t cols) { return 4.0 + (double)rows * (double)cols * 4 / 4e6; }

Plan plan(int dtype, bool direct_a, bool direct_b, bool transposed, int64_t M, int64_t N, int64_t K)
{
    Plan p{choose(dtype, direct_a && direct_b, transposed, M, N, K), false, false};
    if (dtype != TV_BF16 || (direct_a && direct_b) || p.c.kind == kFew || M < 1 || K < 1) return p;
    Choice c = choose(dtype, true, true, M, N, K);
    c.us += (direct_a ? 0.0 : copy_us(M, K)) + (direct_b ? 0.0 : copy_us(N, K));
    return c.us < p.c.us ? Plan{c, !direct_a, !direct_b} : p;
}

int64_t copy_bytes(int64_t rows, int64_t cols) { return up(rows * up(cols, 8) * 2, 256); }

size_t split_bytes(const Choice &c, int64_t M, int64_t N)
{
    return c.splits > 1 ? (size_t)up((int64_t)c.splits * M * up(N, 8) * 4, 256) : 0;
}

bool product_fits(int64_t M, int64_t N) { return tiles(M, 128) * tiles(N, 128) <= kMostTiles; }

int copy_operand(Operand &o, void *to, hipStream_t stream)
{
    const int64_t ld = up(o.cols, 8), units = o.rows * (ld / 8);
    const int64_t groups = tiles(units, 256), wide = (int64_t)1 << 22;
    const dim3 grid = groups <= wide ? dim3((uint32_t)groups) : dim3((uint32_t)wide, (uint32_t)tiles(groups, wide));
    hipLaunchKernelGGL(copy_rows_kernel, grid, dim3(256), 0, stream, (const bf16 *)o.p, o.ld, (bf16 *)to, (int)o.cols, units);
    o = {to, ld, o.rows, ld};
    return launched();
}

template <int BM, int BN, int THREADS>
void launch_tiles(void (*kernel)(Product, Epilogue), Product g, const Epilogue &e, hipStream_t stream)
{
    g.tiles_m = (uint32_t)tiles(g.M, BM);
    g.tiles_n = (uint32_t)tiles(g.N, BN);
    hipLaunchKernelGGL(kernel, dim3(g.tiles_m * g.tiles_n, g.splits), dim3(THREADS), 0, stream, g, e);
}

// NT * 16 columns a workgroup: 16 where 32 would leave half of the compute units without one (2047 -> 513, one row: f32 8.3 us
// with 16, 13.5 with 32; 2048 -> 8192, 16 bf16 rows: 11.4 and 10.1).
template <class T, int NT>
void launch_few(const Product &g, const Epilogue &e, hipStream_t stream)
{
    const dim3 grid((uint32_t)tiles(g.N, NT * 16), g.splits), block(512);
    if (g.M <= 16) hipLaunchKernelGGL((gemv_kernel<T, 1, NT, 8>), grid, block, 0, stream, g, e);
    else if (g.M <= 32) hipLaunchKernelGGL((gemv_kernel<T, 2, NT, 8>), grid, block, 0, stream, g, e);
    else hipLaunchKernelGGL((gemv_kernel<T, 4, NT, 4>), grid, block, 0, stream, g, e);
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
        if (c.kind == kSplit64) launch_tiles<64, 128, 256>(gemm_split_kernel<T, TB, 64, 128, 2, 2, 4, 2, 1, AT, BT>, g, e, stream);
    } else {
        if (c.kind == kSplit256) launch_tiles<256, 256, 512>(gemm_split_kernel<T, TB, 256, 256, 2, 4, 1, 1, 1, AT, BT>, g, e, stream);
        if (c.kind == kSplit128) launch_tiles<128, 128, 512>(gemm_split_kernel<T, TB, 128, 128, 4, 2, 2, 2, 1, AT, BT>, g, e, stream);
        if (c.kind == kSplit64) launch_tiles<64, 128, 512>(gemm_split_kernel<T, TB, 64, 128, 2, 2, 4, 2, 2, AT, BT>, g, e, stream);
    }
    if constexpr (!AT && !BT)
        if (c.kind == kFew) {
            const bool whole_blocks = c.splits == 1 && (e.kind == kHeldBits || e.kind == kHeld8);    // (of 32 columns)
            if (tiles(N, 32) * c.splits > 128 || whole_blocks) launch_few<T, 2>(g, e, stream);
            else launch_few<T, 1>(g, e, stream);
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
    if (d.m < 0 || d.k < 1 || d.n < 1 || d.m >= kMostIndex || d.k >= kMostIndex || d.n >= kMostIndex) return TV_ERR_SHAPE;
    if (!product_fits(d.m, d.n) || !product_fits(d.m, d.k) || !product_fits(d.n, d.k)) return TV_ERR_SHAPE;
    if ((d.dtype != TV_F32 && d.dtype != TV_BF16) || d.act < TV_ACT_NONE || d.act > TV_ACT_SILU) return TV_ERR_UNSUPPORTED;
    if (d.ldx < d.k || d.ldw < d.k || d.ldy < d.n || d.ldx >= kMostStride || d.ldw >= kMostStride || d.ldy >= kMostStride) return TV_ERR_STRIDE;
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

// ---- the forward call's workspace: copies of x and W, split sums
struct FwdPlan {
    Plan product;
    size_t w, split, bytes;
};

FwdPlan fwd_plan(const tv_linear_desc &d, bool direct_x, bool direct_w)
{
    FwdPlan p{};
    p.product = plan(d.dtype, direct_x, direct_w, false, d.m, d.n, d.k);
    p.w = p.product.copy_a ? copy_bytes(d.m, d.k) : 0;
    p.split = p.w + (p.product.copy_b ? copy_bytes(d.n, d.k) : 0);
    p.bytes = p.split + split_bytes(p.product.c, d.m, d.n);
    return p;
}

template <class T>
int linear_fwd(const void *x, const void *w, const void *bias, const void *res, void *y, const tv_held &h,
               const tv_linear_desc &d, const FwdPlan &p, char *ws, hipStream_t stream)
{
    Epilogue e{};
    e.bias = bias; e.res = res; e.y = y;
    e.held = h.kind == TV_HELD_NONE ? nullptr : h.data; e.exps = h.exps;
    e.ldr = d.ldr; e.ldy = d.ldy; e.act = d.act; e.kind = h.kind;
    Operand a{x, d.ldx, d.m, d.k}, b{w, d.ldw, d.n, d.k};
    if (p.product.copy_a && copy_operand(a, ws, stream) != TV_OK) return TV_ERR_HIP;
    if (p.product.copy_b && copy_operand(b, ws + p.w, stream) != TV_OK) return TV_ERR_HIP;
    return run_product<T, T, false, false>(a, b, d.m, d.n, d.k, p.product.c, e, ws + p.split, stream);
}

// ---- the backward call's workspace: dz (or a copy of g), x out of its checkpoint or a copy of it, a copy of W, the column
// sums of groups of rows, split sums
struct BwdPlan {
    Plan dx, dw;
    size_t x, w, sums, split, bytes;
    int64_t ldz, ldx;
    int rows_per, groups;
    bool own_dz, own_x;
};

BwdPlan bwd_plan(const tv_linear_desc &d, bool x8, bool direct_g, bool direct_x, bool direct_w)
{
    BwdPlan p{};
    const int64_t size = (int64_t)elem_bytes(d.dtype);
    const bool smooth = d.act != TV_ACT_NONE;
    // dz is written, and codes are restored, into rows that go straight to LDS
    p.dx = plan(d.dtype, smooth || direct_g, direct_w, true, d.m, d.k, d.n);
    p.dw = plan(d.dtype, smooth || direct_g, x8 || direct_x, true, d.n, d.k, d.m);
    p.own_dz = smooth || p.dx.copy_a || p.dw.copy_a;
    p.own_x = x8 || p.dw.copy_b;
    p.ldz = up(d.n, 8);
    p.ldx = up(d.k, 8);
    size_t at = p.own_dz ? up(d.m * p.ldz * size, 256) : 0;
    p.x = at;
    if (p.own_x) at += copy_bytes(d.m, d.k);
    p.w = at;
    if (p.dx.copy_b) at += copy_bytes(d.n, d.k);
    // about 1024 workgroups of 256 columns each, of sixteen rows at least; up to 64 rows are one group, one launch
    const int64_t want = 1024 / tiles(d.n, 256) + 1;
    p.rows_per = (int)(d.m > 64 ? up(tiles(d.m, want < 256 ? want : 256), 16) : 64);
    p.groups = (int)tiles(d.m, p.rows_per);
    p.sums = at;
    at += up((int64_t)p.groups * d.n * 4, 256);
    p.split = at;
    const size_t s1 = split_bytes(p.dx.c, d.m, d.k), s2 = split_bytes(p.dw.c, d.n, d.k);
    p.bytes = at + (s1 > s2 ? s1 : s2);
    return p;
}

template <class T>
int linear_bwd(const void *g, const void *x, const uint8_t *x_exps, const tv_held &h, const void *w, void *dx, void *dw,
               void *db, const tv_linear_desc &d, const BwdPlan &p, char *ws, hipStream_t stream)
{
    Operand dz{g, d.ldy, d.m, d.n};
    const bool own_dz = d.act != TV_ACT_NONE || (dx && p.dx.copy_a) || (dw && p.dw.copy_a);
    if (d.m > 0 && (own_dz || db)) {
        SlopeArgs a{};
        a.g = g; a.held = h.data; a.exps = h.exps;
        a.dz = own_dz ? ws : nullptr;
        a.sums = db && p.groups > 1 ? (float *)(ws + p.sums) : nullptr;
        a.db = p.groups == 1 ? db : nullptr;
        a.ldg = d.ldy; a.ldz = p.ldz;
        a.M = (int32_t)d.m; a.N = (int32_t)d.n; a.rows_per = p.rows_per;
        a.act = d.act; a.kind = d.act == TV_ACT_NONE ? TV_HELD_NONE : h.kind;
        hipLaunchKernelGGL((slope_kernel<T>), dim3((uint32_t)tiles(d.n, 256), p.groups), dim3(256), 0, stream, a);
        if (launched() != TV_OK) return TV_ERR_HIP;
        if (own_dz) dz = {ws, p.ldz, d.m, p.ldz};
    }
    if (db && p.groups != 1) {
        hipLaunchKernelGGL((column_sum_kernel<T>), dim3((uint32_t)tiles(d.n, 32)), dim3(256), 0, stream,
                           (const float *)(ws + p.sums), (T *)db, d.m > 0 ? p.groups : 0, (int)d.n);
        if (launched() != TV_OK) return TV_ERR_HIP;
    }
    if (dx && d.m > 0) {
        Operand b{w, d.ldw, d.n, d.k};
        if (p.dx.copy_b && copy_operand(b, ws + p.w, stream) != TV_OK) return TV_ERR_HIP;
        const int st = run_product<T, T, false, true>(dz, b, d.m, d.k, d.n, p.dx.c, plain_output(dx, d.k), ws + p.split, stream);
        if (st != TV_OK) return st;
    }
    if (dw) {
        Operand b{x, d.ldx, d.m, d.k};
        if (x_exps && d.m > 0) {                      // what codes stand for is exact in bf16
            const int st = tv_ckpt8_load((const int8_t *)x, x_exps, ws + p.x, d.m, d.k, p.ldx, TV_BF16, stream);
            if (st != TV_OK) return st;
            b = {ws + p.x, p.ldx, d.m, p.ldx};
        } else if (p.dw.copy_b && copy_operand(b, ws + p.x, stream) != TV_OK) return TV_ERR_HIP;
        const Epilogue e = plain_output(dw, d.k);
        return x_exps ? run_product<T, bf16, true, true>(dz, b, d.n, d.k, d.m, p.dw.c, e, ws + p.split, stream)
                      : run_product<T, T, true, true>(dz, b, d.n, d.k, d.m, p.dw.c, e, ws + p.split, stream);
    }
    return TV_OK;
}

int check_ckpt8(int64_t rows, int64_t n, int64_t ld, int dtype)
{
    if (rows < 0 || n < 1 || rows >= kMostIndex || n >= kMostIndex) return TV_ERR_SHAPE;
    if (rows > ((int64_t)1 << 40) / n) return TV_ERR_SHAPE;
    if (dtype != TV_F32 && dtype != TV_BF16) return TV_ERR_UNSUPPORTED;
    if (ld < n || ld >= kMostStride) return TV_ERR_STRIDE;
    return TV_OK;
}

dim3 ckpt8_grid(int64_t rows, int64_t n)
{
    const int64_t groups = tiles(rows * tiles(n, kBlock), 64), wide = (int64_t)1 << 22;
    return groups <= wide ? dim3((uint32_t)groups) : dim3((uint32_t)wide, (uint32_t)tiles(groups, wide));
}

}  // namespace

extern "C" {

// (The workspaces are asked for before there are pointers, and have to do wherever those lie.)
size_t tv_linear_fwd_workspace_bytes(tv_linear_desc d)
{
    size_t most = 0;
    if (check_sizes(d) == TV_OK && d.m > 0)
        for (int i = 0; i < 4; ++i) {
            const size_t b = fwd_plan(d, (i & 1) != 0, (i & 2) != 0).bytes;
            most = most > b ? most : b;
        }
    return most;
}

int tv_linear_fwd(const void *x, const void *w, const void *bias, const void *res, void *y, tv_held held,
                  tv_linear_desc d, void *ws, size_t ws_bytes, hipStream_t stream)
{
    int st = check_sizes(d);
    if (st != TV_OK) return st;
    if (res && (d.ldr < d.n || d.ldr >= kMostStride)) return TV_ERR_STRIDE;
    if ((st = check_held(d, held, false)) != TV_OK) return st;
    if (d.m == 0) return TV_OK;
    if (!x || !w || !y) return TV_ERR_NULL;
    const size_t size = elem_bytes(d.dtype);
    if (!aligned(x, size) || !aligned(w, size) || !aligned(bias, size) || !aligned(res, size) || !aligned(y, size)) return TV_ERR_STRIDE;
    const FwdPlan p = fwd_plan(d, direct({x, d.ldx, d.m, d.k}), direct({w, d.ldw, d.n, d.k}));
    if ((st = check_workspace(ws, ws_bytes, p.bytes)) != TV_OK) return st;
    return d.dtype == TV_BF16 ? linear_fwd<bf16>(x, w, bias, res, y, held, d, p, (char *)ws, stream)
                              : linear_fwd<float>(x, w, bias, res, y, held, d, p, (char *)ws, stream);
}

size_t tv_linear_bwd_workspace_bytes(tv_linear_desc d, int x_is_8bit)
{
    size_t most = 0;
    if (check_sizes(d) == TV_OK)
        for (int i = 0; i < 8; ++i) {
            const size_t b = bwd_plan(d, x_is_8bit != 0, (i & 1) != 0, (i & 2) != 0, (i & 4) != 0).bytes;
            most = most > b ? most : b;
        }
    return most;
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
    const BwdPlan p = bwd_plan(d, x_exps != nullptr, direct({g, d.ldy, d.m, d.n}), direct({x, d.ldx, d.m, d.k}), direct({w, d.ldw, d.n, d.k}));
    if ((st = check_workspace(ws, ws_bytes, p.bytes)) != TV_OK) return st;
    return d.dtype == TV_BF16 ? linear_bwd<bf16>(g, x, x_exps, held, w, dx, dw, db, d, p, (char *)ws, stream)
                              : linear_bwd<float>(g, x, x_exps, held, w, dx, dw, db, d, p, (char *)ws, stream);
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
