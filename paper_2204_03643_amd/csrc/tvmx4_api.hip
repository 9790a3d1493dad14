// C-ABI entry points of values in 4 bits and their products: argument validation and launches.
#include "../../include/tvprox.h"
#include "tv_gemm4.hpp"
#include "tv_linear_plan.hpp"

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

// 16 rows by a group a workgroup; beyond 65536 by 64 they take further ones in turn
dim3 values_grid(int64_t rows, int64_t n)
{
    const int64_t x = tiles(rows, 16), y = groups4(n);
    return dim3((uint32_t)(x < 65536 ? x : 65536), (uint32_t)(y < 64 ? y : 64));
}

template <class T>
int save(const void *x, void *codes, void *exps, int64_t rows, int64_t n, int64_t ldx, hipStream_t stream)
{
    hipLaunchKernelGGL((mx4_save_kernel<T>), values_grid(rows, n), dim3(256), 0, stream, (const T *)x, ldx, (uint8_t *)codes, (uint32_t *)exps, rows, (int)n, (int)groups4(n));
    return launched();
}

int check_sizes(const tv_linear_desc &d, bool codes)
{
    if (d.m < 0 || d.k < 1 || d.n < 1 || d.m >= kMostIndex || d.k >= kMostIndex || d.n >= kMostIndex) return TV_ERR_SHAPE;
    if (!product_fits(d.m, d.n)) return TV_ERR_SHAPE;
    if ((d.dtype != TV_F32 && d.dtype != TV_BF16) || d.act < TV_ACT_NONE || d.act > TV_ACT_SILU) return TV_ERR_UNSUPPORTED;
    if (d.ldy < d.n || d.ldy >= kMostStride || (!codes && (d.ldx < d.k || d.ldx >= kMostStride))) return TV_ERR_STRIDE;
    return TV_OK;
}

// The workspace: x's codes and scale words.
struct Plan4 {
    size_t exps, bytes;
};
Plan4 plan4(const tv_linear_desc &d, bool codes)
{
    Plan4 p{};
    if (!codes) {
        p.exps = (size_t)up(d.m * groups4(d.k) * 64, 256);
        p.bytes = p.exps + (size_t)up(rows4(d.m) * groups4(d.k) * 4, 256);
    }
    return p;
}

template <class T>
int linear4(const void *x, const uint8_t *x_exps, const uint8_t *w, const uint8_t *w_exps, const Epilogue &e,
            const tv_linear_desc &d, const Plan4 &p, char *ws, hipStream_t stream)
{
    Product4 g{(const uint8_t *)x, w, (const uint32_t *)x_exps, (const uint32_t *)w_exps, (int32_t)d.m, (int32_t)d.n, (int32_t)groups4(d.k)};
    if (!x_exps) {
        if (save<T>(x, ws, ws + p.exps, d.m, d.k, d.ldx, stream) != TV_OK) return TV_ERR_HIP;
        g.x = (const uint8_t *)ws;
        g.xs = (const uint32_t *)(ws + p.exps);
    }
    hipLaunchKernelGGL((linear4_kernel<T>), dim3((uint32_t)(tiles(d.n, 64) * tiles(d.m, 32))), dim3(256), 0, stream, g, e);
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
        hipLaunchKernelGGL((mx4_load_kernel<bf16>), values_grid(rows, n), dim3(256), 0, stream, codes, exps, (bf16 *)x, ldx, rows, (int)n, (int)groups4(n));
    else
        hipLaunchKernelGGL((mx4_load_kernel<float>), values_grid(rows, n), dim3(256), 0, stream, codes, exps, (float *)x, ldx, rows, (int)n, (int)groups4(n));
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
