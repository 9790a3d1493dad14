// C-ABI entry points of the channel products and the 8-bit checkpoints: argument validation and launches.
#include "../../include/tvprox.h"
#include "tv_ckpt8.hpp"
#include "tv_gemm_split.hpp"
#include "tv_gemv.hpp"
#include "tv_linear_plan.hpp"
#include "tv_slope.hpp"

namespace {

using namespace tvl;

int launched() { return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP; }

// ---- products
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

template <class T>
int linear_bwd(const void *g, const void *x, const uint8_t *x_exps, const tv_held &h, const void *w, void *dx, void *dw,
               void *db, const tv_linear_desc &d, const BwdPlan &p, char *ws, hipStream_t stream)
{
    Operand dz{g, d.ldy, d.m, d.n};
    if (d.m > 0 && (p.own_dz || db)) {
        SlopeArgs a{};
        a.g = g; a.held = h.data; a.exps = h.exps;
        a.dz = p.own_dz ? ws : nullptr;
        a.sums = db && p.groups > 1 ? (float *)(ws + p.sums) : nullptr;
        a.db = p.groups == 1 ? db : nullptr;
        a.ldg = d.ldy; a.ldz = p.ldz;
        a.M = (int32_t)d.m; a.N = (int32_t)d.n; a.rows_per = p.rows_per;
        a.act = d.act; a.kind = d.act == TV_ACT_NONE ? TV_HELD_NONE : h.kind;
        hipLaunchKernelGGL((slope_kernel<T>), dim3((uint32_t)tiles(d.n, 256), p.groups), dim3(256), 0, stream, a);
        if (launched() != TV_OK) return TV_ERR_HIP;
        if (p.own_dz) dz = {ws, p.ldz, d.m, p.ldz};
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

// The plans of calls with these pointers, of which alignments count, and whether outputs are there at all.
FwdPlan fwd_plan_of(const void *x, const void *w, const tv_linear_desc &d)
{
    return fwd_plan(d, direct({x, d.ldx, d.m, d.k}), direct({w, d.ldw, d.n, d.k}));
}
BwdPlan bwd_plan_of(const void *g, const void *x, const uint8_t *x_exps, const void *w, const void *dx, const void *dw, const void *db, const tv_linear_desc &d)
{
    return bwd_plan(d, x_exps != nullptr, direct({g, d.ldy, d.m, d.n}), direct({x, d.ldx, d.m, d.k}), direct({w, d.ldw, d.n, d.k}),
                    {dx != nullptr, dw != nullptr, db != nullptr});
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

// (The workspaces that are asked for without pointers have to do wherever those lie.)
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

size_t tv_linear_fwd_workspace_bytes_at(const void *x, const void *w, tv_linear_desc d)
{
    return check_sizes(d) == TV_OK && d.m > 0 ? fwd_plan_of(x, w, d).bytes : 0;
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
    const FwdPlan p = fwd_plan_of(x, w, d);
    if ((st = check_workspace(ws, ws_bytes, p.bytes)) != TV_OK) return st;
    return d.dtype == TV_BF16 ? linear_fwd<bf16>(x, w, bias, res, y, held, d, p, (char *)ws, stream)
                              : linear_fwd<float>(x, w, bias, res, y, held, d, p, (char *)ws, stream);
}

size_t tv_linear_bwd_workspace_bytes(tv_linear_desc d, int x_is_8bit)
{
    size_t most = 0;
    if (check_sizes(d) == TV_OK)
        for (int i = 0; i < 8; ++i) {
            const size_t b = bwd_plan(d, x_is_8bit != 0, (i & 1) != 0, (i & 2) != 0, (i & 4) != 0, {true, true, true}).bytes;
            most = most > b ? most : b;
        }
    return most;
}

size_t tv_linear_bwd_workspace_bytes_at(const void *g, const void *x, const uint8_t *x_exps, const void *w, const void *dx,
                                        const void *dw, const void *db, tv_linear_desc d)
{
    return check_sizes(d) == TV_OK ? bwd_plan_of(g, x, x_exps, w, dx, dw, db, d).bytes : 0;
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
    const BwdPlan p = bwd_plan_of(g, x, x_exps, w, dx, dw, db, d);
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
