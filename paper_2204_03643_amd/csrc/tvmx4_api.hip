// C-ABI entry points of values in 4 bits and their products: argument validation and launches.
#include "../../include/tvprox.h"
#include "tv_gemv4.hpp"
#include "tv_linear4_plan.hpp"

namespace {

using namespace tvl;

int launched() { return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP; }

int check_values(int64_t rows, int64_t n, int64_t ld, int dtype)
{
    if (rows < 0 || n < 1 || rows >= kMostIndex || n >= kMostIndex) return TV_ERR_SHAPE;
    if (rows > ((int64_t)1 << 40) / n) return TV_ERR_SHAPE;
    if (dtype != TV_F32 && dtype != TV_BF16) return TV_ERR_UNSUPPORTED;
    if (ld < n || ld >= kMostStride) return TV_ERR_STRIDE;
    return TV_OK;
}

// `each` groups by 16 rows a workgroup; beyond 64 by 65535 they take further ones in turn
dim3 values_grid(int64_t rows, int64_t n, int each)
{
    const int64_t x = tiles(groups4(n), each), y = tiles(rows, 16);
    return dim3((uint32_t)(x < 64 ? x : 64), (uint32_t)(y < 65535 ? y : 65535));
}

// One group at a time where four would leave compute units without a workgroup (64 x 8192: 2.8 us with one, 4.2 with four;
// 8192 x 2048: 13.1 and 9.8).
template <class T>
int save(const void *x, void *codes, void *exps, int64_t rows, int64_t n, int64_t ldx, hipStream_t stream)
{
    const int groups = (int)groups4(n);
    if (tiles(rows, 16) * tiles(groups, 4) >= 1024)
        hipLaunchKernelGGL((mx4_save_kernel<T, 4>), values_grid(rows, n, 4), dim3(256), 0, stream, (const T *)x, ldx, (uint8_t *)codes, (uint32_t *)exps, rows, (int)n, groups);
    else
        hipLaunchKernelGGL((mx4_save_kernel<T, 1>), values_grid(rows, n, 1), dim3(256), 0, stream, (const T *)x, ldx, (uint8_t *)codes, (uint32_t *)exps, rows, (int)n, groups);
    return launched();
}

int check_sizes(const tv_linear_desc &d, bool codes)
{
    if (d.m < 0 || d.k < 1 || d.n < 1 || d.m >= kMostIndex || d.k >= kMostIndex || d.n >= kMostIndex) return TV_ERR_SHAPE;
    if (!product_fits(d.m, d.n)) return TV_ERR_SHAPE;
    if (d.k > TV_LINEAR4_MAX_K) return TV_ERR_UNSUPPORTED;
    if ((d.dtype != TV_F32 && d.dtype != TV_BF16) || d.act < TV_ACT_NONE || d.act > TV_ACT_SILU) return TV_ERR_UNSUPPORTED;
    if (d.ldy < d.n || d.ldy >= kMostStride || (!codes && (d.ldx < d.k || d.ldx >= kMostStride))) return TV_ERR_STRIDE;
    return TV_OK;
}

template <class T, int BM, int BN, int WM, int WN, int BUF, int G>
void launch_tiles(Product g, const Scales &scales, const Epilogue &e, hipStream_t stream)
{
    g.tiles_m = (uint32_t)tiles(g.M, BM);
    g.tiles_n = (uint32_t)tiles(g.N, BN);
    hipLaunchKernelGGL((gemm4_kernel<T, BM, BN, WM, WN, BUF, G>), dim3(g.tiles_m * g.tiles_n, g.splits), dim3(WM * WN * 64), 0, stream, g, scales, e);
}

template <class T, int NT>
void launch_few(const Product &g, const Rows4 &x, bool own, const Scales &s, const Epilogue &e, hipStream_t stream)
{
    const dim3 grid((uint32_t)tiles(g.N, 16 * NT)), block(512);
    if (own) hipLaunchKernelGGL((gemv4_kernel<T, 1, NT, 2, true>), grid, block, 0, stream, g, x, s.w, s.w_rows, e);
    else if (g.M <= 16) hipLaunchKernelGGL((gemv4_kernel<T, 1, NT, 4, false>), grid, block, 0, stream, g, x, s.w, s.w_rows, e);
    else hipLaunchKernelGGL((gemv4_kernel<T, 2, NT, 4, false>), grid, block, 0, stream, g, x, s.w, s.w_rows, e);
}

template <class T>
int linear4(const void *x, const uint8_t *x_exps, const uint8_t *w, const uint8_t *w_exps, const Epilogue &e,
            const tv_linear_desc &d, const Plan4 &p, char *ws, hipStream_t stream)
{
    const int64_t ld = groups_of(d.k) * 32;
    Product g{x, w, ld, ld, (int32_t)d.m, (int32_t)d.n, (int32_t)ld, p.c.k_per, p.c.splits, (float *)(ws + p.split), 0, 0};
    const Scales s{p.c.own ? nullptr : x_exps ? (const uint32_t *)x_exps : (const uint32_t *)(ws + p.exps), (const uint32_t *)w_exps,
                   (uint32_t)scale_rows(d.m), (uint32_t)scale_rows(d.n)};
    if (!x_exps && !p.c.own) {
        if (save<T>(x, ws, ws + p.exps, d.m, d.k, d.ldx, stream) != TV_OK) return TV_ERR_HIP;
        g.a = ws;
    }
    if (p.c.kind == kTile256x4) launch_tiles<T, 256, 256, 2, 4, 2, 2>(g, s, e, stream);
    if (p.c.kind == kTile128x4) launch_tiles<T, 128, 128, 2, 2, 4, 2>(g, s, e, stream);
    if (p.c.kind == kTile64x4) launch_tiles<T, 64, 128, 2, 2, 4, 2>(g, s, e, stream);
    if (p.c.kind == kFew4) {
        const Rows4 rows{g.a, s.x, d.ldx, s.x_rows, (int32_t)d.k};
        // The fewest columns a workgroup with which no compute unit has two of them, 64 at most.  One row of 4096 in bf16 with 16, 32
        // and 64, us in a graph: -> 4096 5.3, 5.6, 7.5; 4104 6.9, 5.5, 7.4; 8192 7.6, 5.6, 7.6; 8200 9.3, 8.0, 7.7; 16384 13.7, 9.5,
        // 7.9.  With codes there is nothing of x to share, and the same rule loses at most 2: 4104 4.2, 4.7, 6.4; 8200 5.5, 6.0,
        // 7.4; 16384 8.5, 7.5, 7.9; 32 rows of them 7.5, 6.3, 8.4; 10.4, 9.2, 9.2; 14.5, 10.5, 9.5.
        if (d.n > 8192) launch_few<T, 4>(g, rows, p.c.own, s, e, stream);
        else if (d.n > 4096) launch_few<T, 2>(g, rows, p.c.own, s, e, stream);
        else launch_few<T, 1>(g, rows, p.c.own, s, e, stream);
    }
    if (p.c.splits > 1) {
        if (launched() != TV_OK) return TV_ERR_HIP;
        hipLaunchKernelGGL((join_kernel<T>), dim3((uint32_t)tiles(d.m * tiles(d.n, 32) * 4, 256)), dim3(256), 0, stream, g, e);
    }
    return launched();
}

}  // namespace

extern "C" {

int tv_mx4_save(const void *x, uint8_t *codes, uint8_t *exps, int64_t rows, int64_t n, int64_t ldx, int dtype, hipStream_t stream)
{
    const int st = check_values(rows, n, ldx, dtype);
    if (st != TV_OK || rows == 0) return st;
    if (!x || !codes || !exps) return TV_ERR_NULL;
    if (!aligned(x, elem_bytes(dtype)) || !aligned(codes, 16) || !aligned(exps, 16)) return TV_ERR_STRIDE;
    return dtype == TV_BF16 ? save<bf16>(x, codes, exps, rows, n, ldx, stream) : save<float>(x, codes, exps, rows, n, ldx, stream);
}

int tv_mx4_load(const uint8_t *codes, const uint8_t *exps, void *x, int64_t rows, int64_t n, int64_t ldx, int dtype, hipStream_t stream)
{
    const int st = check_values(rows, n, ldx, dtype);
    if (st != TV_OK || rows == 0) return st;
    if (!x || !codes || !exps) return TV_ERR_NULL;
    if (!aligned(x, elem_bytes(dtype)) || !aligned(codes, 16) || !aligned(exps, 16)) return TV_ERR_STRIDE;
    if (dtype == TV_BF16)
        hipLaunchKernelGGL((mx4_load_kernel<bf16>), values_grid(rows, n, 1), dim3(256), 0, stream, codes, exps, (bf16 *)x, ldx, rows, (int)n, (int)groups4(n));
    else
        hipLaunchKernelGGL((mx4_load_kernel<float>), values_grid(rows, n, 1), dim3(256), 0, stream, codes, exps, (float *)x, ldx, rows, (int)n, (int)groups4(n));
    return launched();
}

size_t tv_linear4_workspace_bytes(tv_linear_desc d, int x_is_codes)
{
    return check_sizes(d, x_is_codes != 0) == TV_OK && d.m > 0 ? plan4(d, x_is_codes != 0).bytes : 0;
}

int tv_linear4_fwd(const void *x, const uint8_t *x_exps, const uint8_t *w, const uint8_t *w_exps, const void *bias,
                   const void *res, void *y, tv_linear_desc d, void *ws, size_t ws_bytes, hipStream_t stream)
{
    const int st = check_sizes(d, x_exps != nullptr);
    if (st != TV_OK) return st;
    if (res && (d.ldr < d.n || d.ldr >= kMostStride)) return TV_ERR_STRIDE;
    if (d.m == 0) return TV_OK;
    if (!x || !w || !w_exps || !y) return TV_ERR_NULL;
    const size_t size = elem_bytes(d.dtype);
    if (!aligned(x, x_exps ? 16 : size) || !aligned(x_exps, 16) || !aligned(w, 16) || !aligned(w_exps, 16)) return TV_ERR_STRIDE;
    if (!aligned(bias, size) || !aligned(res, size) || !aligned(y, size)) return TV_ERR_STRIDE;
    const Plan4 p = plan4(d, x_exps != nullptr);
    if (p.bytes && (!ws || !aligned(ws, 16) || ws_bytes < p.bytes)) return TV_ERR_WORKSPACE;
    Epilogue e{};
    e.bias = bias; e.res = res; e.y = y;
    e.ldr = d.ldr; e.ldy = d.ldy; e.act = d.act; e.kind = kHeldNone;
    return d.dtype == TV_BF16 ? linear4<bf16>(x, x_exps, w, w_exps, e, d, p, (char *)ws, stream)
                              : linear4<float>(x, x_exps, w, w_exps, e, d, p, (char *)ws, stream);
}

}  // extern "C"
