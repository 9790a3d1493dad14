// Products of values in 4 bits: D[m, n] = sum_k X(m, k) W(n, k), both in blocks of 32 with a scale each.
#pragma once
#include "tv_gemm.hpp"
#include "tv_mx4.hpp"

namespace tvl {

typedef int32_t s32x8 __attribute__((ext_vector_type(8)));

struct Product4 {
    const uint8_t  *x, *w;          // codes, 64 bytes a group of a row
    const uint32_t *xs, *ws;        // scale words [groups, rows up to a multiple of four]
    int32_t M, N, groups;
};

__device__ __forceinline__ s32x8 operand4(u32x4 v)
{
    return s32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}

// 32 rows of x by 64 of W a workgroup, 16 of W a wave: operands straight from memory.
template <class T> __global__ __launch_bounds__(256) void linear4_kernel(Product4 g, Epilogue e)
{
    __shared__ __attribute__((aligned(16))) float out[32 * kOutPitch];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, block = lane >> 4;
    const uint32_t columns = ((uint32_t)g.N + 63) / 64;
    const int m0 = (int)(blockIdx.x / columns) * 32, n0 = (int)(blockIdx.x % columns) * 64;
    const int n = min(n0 + wave * 16 + r, g.N - 1), m[2] = {min(m0 + r, g.M - 1), min(m0 + 16 + r, g.M - 1)};
    f32x4 acc[2] = {};
    for (int k = 0; k < g.groups; ++k) {
        const u32x4 w = *(const u32x4 *)(g.w + ((int64_t)n * g.groups + k) * 64 + block * 16);
        const int ws = (int)(g.ws[k * rows4(g.N) + n] >> (8 * block));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4 x = *(const u32x4 *)(g.x + ((int64_t)m[i] * g.groups + k) * 64 + block * 16);
            const int xs = (int)(g.xs[k * rows4(g.M) + m[i]] >> (8 * block));
            acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand4(w), operand4(x), acc[i], 4, 4, 0, ws, 0, xs);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) *(f32x4 *)&out[(16 * i + r) * kOutPitch + wave * 16 + block * 4] = acc[i];
    __syncthreads();
    const int row = threadIdx.x >> 3, col = (threadIdx.x & 7) * 8;
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = out[row * kOutPitch + col + i];
    finish8<T>(p, m0 + row, n0 + col, g.N, m0 + row < g.M, e);
}

}  // namespace tvl
