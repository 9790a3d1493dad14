// dz = g act'(z) from what the forward call held of z, and the column sums of dz (the bias gradient), in one pass.
#pragma once
#include "tv_linear.hpp"

namespace tvl {

struct SlopeArgs {
    const void    *g;          // [M, N] rows of ldg elements
    const void    *held;       // z as the forward call held it
    const uint8_t *exps;
    void          *dz;         // [M, N] rows of ldz elements, or null (the column sums alone)
    float         *sums;       // [groups of rows, N] column sums, or null
    int64_t        ldg, ldz;
    int32_t        M, N, rows_per;
    int32_t        act, kind;
    uint32_t       vec;
};

// Four columns a thread, 64 threads a row, four rows at a time; `rows_per` rows a workgroup.
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a)
{
    constexpr bool kFast = sizeof(T) == 2;
    __shared__ f32x4 part[3][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n = ((int)blockIdx.x * 64 + lane) * 4, have = max(0, min(4, a.N - n));
    const int blocks = (a.N + 31) / 32;
    const int64_t first = (int64_t)blockIdx.y * a.rows_per, last = min((int64_t)a.M, first + a.rows_per);
    const bool vec = a.vec != 0;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (have)
        for (int64_t m = first + wave; m < last; m += 4) {
            f32x4 d = load4((const T *)a.g + m * a.ldg + n, have, vec);
            if (a.kind == kHeldBits) {
                const uint32_t w = ((const uint32_t *)a.held)[m * blocks + n / 32] >> (n & 31);
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] = (w >> i) & 1u ? d[i] : 0.0f;
            } else if (a.kind == kHeldPlain) {
                const f32x4 z = load4((const T *)a.held + m * a.N + n, have, vec);
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] *= slope_of<kFast>(z[i], a.act);
            } else if (a.kind == kHeld8) {
                const uint32_t byte = a.exps[m * blocks + n / 32];
                const int8_t *from = (const int8_t *)a.held + m * a.N + n;
                uint32_t c = 0;
                if (have == 4 && vec) c = *(const uint32_t *)from;
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < have) c |= (uint32_t)(uint8_t)from[i] << (8 * i);
#pragma unroll
                for (int i = 0; i < 4; ++i) d[i] *= slope_of<kFast>(value_of((int)(int8_t)(c >> (8 * i)), byte), a.act);
            }
            if (a.dz) store4((T *)a.dz + m * a.ldz + n, d, have, vec);
            sum += d;
        }
    if (!a.sums) return;
    if (wave) part[wave - 1][lane] = sum;
    __syncthreads();
    if (wave == 0 && have) {
        sum = ((sum + part[0][lane]) + part[1][lane]) + part[2][lane];
        float *to = a.sums + (int64_t)blockIdx.y * a.N + n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) to[i] = sum[i];
    }
}

// The bias gradient from the groups' sums, always in the same order: 32 columns a workgroup, eight threads a column.
template <class T>
__global__ __launch_bounds__(256) void column_sum_kernel(const float *sums, T *db, int groups, int N)
{
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, share = threadIdx.x >> 5, n = (int)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (n < N)
#pragma unroll 8
        for (int i = share; i < groups; i += 8) s += sums[(int64_t)i * N + n];
    part[share][lane] = s;
    __syncthreads();
    if (share == 0 && n < N) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i][lane];
        db[n] = narrow<T>(s);
    }
}

}  // namespace tvl
