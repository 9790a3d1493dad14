// dz = g act'(z) from what the forward call held of z, and the column sums of dz (the bias gradient), in one pass.
//
// dz leaves in the call's dtype.  In bf16 that rounds it once more before the products that give dx and dW, which take bf16
// operands: their 2-norm is off by 1.7e-3 for it, as much as for their own rounding (2.4e-3 together).  A second bf16 part
// would take that away and double both products.  The column sums are of dz before it is rounded.
#pragma once
#include "tv_linear.hpp"

namespace tvl {

struct SlopeArgs {
    const void    *g;          // [M, N] rows of ldg elements
    const void    *held;       // z as the forward call held it
    const uint8_t *exps;
    void          *dz;         // [M, ldz], rows on 16-byte boundaries, zeros past N; or null (the column sums alone)
    float         *sums;       // [groups of rows, N] column sums, or null
    void          *db;         // [N] column sums of all rows (where one group holds them), or null
    int64_t        ldg, ldz;
    int32_t        M, N, rows_per;
    int32_t        act, kind;
};

// Eight columns a thread, 32 threads a row, eight rows at a time; `rows_per` rows a workgroup, two of a thread's rows on
// their way together (what is read and written bounds the kernel where enough is in flight: 8192 x 8192 bf16 with gelu
// moves 403 MB in 91 us, 4.4 TB/s).
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a)
{
    constexpr bool kFast = sizeof(T) == 2;
    constexpr int kRows = 8, kRaw = sizeof(T) / 2, kAhead = 2;
    __shared__ float part[kRows - 1][32][9];
    const int lane = threadIdx.x & 31, share = threadIdx.x >> 5;
    const int n = ((int)blockIdx.x * 32 + lane) * 8, have = max(0, min(8, a.N - n));
    const int blocks = (a.N + 31) / 32;
    const int64_t first = (int64_t)blockIdx.y * a.rows_per, last = min((int64_t)a.M, first + a.rows_per);
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};

    auto slopes = [&](float (&d)[8], const float (&z)[8]) {
        if (a.act == kGelu)
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= slope_of<kFast>(z[i], kGelu);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= slope_of<kFast>(z[i], kSilu);
    };
    auto row = [&](int64_t m, float (&d)[8], uint32_t word, uint32_t byte, const u32x4 (&z)[kRaw], u32x2 code) {
        if (a.kind == kHeldBits) {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = (word >> i) & 1u ? d[i] : 0.0f;
        } else if (a.kind == kHeldPlain) {
            float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            add8<T>(v, z);
            slopes(d, v);
        } else if (a.kind == kHeld8) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = value_of((int)(int8_t)(code[i >> 2] >> (8 * (i & 3))), byte);
            slopes(d, v);
        }
        if (a.dz) store8((T *)a.dz + m * a.ldz + n, d, 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += d[i];
    };
    if (have == 8) {
        for (int64_t m = first + share; m < last; m += kRows * kAhead) {
            u32x4 g[kAhead][kRaw], z[kAhead][kRaw];
            u32x2 code[kAhead];
            uint32_t word[kAhead], byte[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int64_t r = min(m + u * kRows, last - 1);
#pragma unroll
                for (int j = 0; j < kRaw; ++j) g[u][j] = get16((const T *)a.g + r * a.ldg + n + j * (16 / (int)sizeof(T)));
                if (a.kind == kHeldPlain)
#pragma unroll
                    for (int j = 0; j < kRaw; ++j) z[u][j] = get16((const T *)a.held + r * a.N + n + j * (16 / (int)sizeof(T)));
                if (a.kind == kHeldBits) word[u] = ((const uint32_t *)a.held)[r * blocks + n / 32] >> (n & 31);
                if (a.kind == kHeld8) {
                    code[u] = *(const u32x2_at1 *)((const int8_t *)a.held + r * a.N + n);
                    byte[u] = a.exps[r * blocks + n / 32];
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (m + u * kRows < last) {
                    float d[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                    add8<T>(d, g[u]);
                    row(m + u * kRows, d, word[u], byte[u], z[u], code[u]);
                }
        }
    } else if (have) {
        for (int64_t m = first + share; m < last; m += kRows) {
            float d[8], v[8];
            load8(d, (const T *)a.g + m * a.ldg + n, have);
            uint32_t word = 0, byte = 1;
            u32x2 code = {0, 0};
            u32x4 z[kRaw] = {};
            if (a.kind == kHeldBits) word = ((const uint32_t *)a.held)[m * blocks + n / 32] >> (n & 31);
            if (a.kind == kHeldPlain) {
                load8(v, (const T *)a.held + m * a.N + n, have);
                if constexpr (sizeof(T) == 2) {
                    bf16x8 h;
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[i] = narrow<bf16>(v[i]);       // (exact: they were bf16)
                    z[0] = __builtin_bit_cast(u32x4, h);
                } else {
                    z[0] = __builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]});
                    z[kRaw - 1] = __builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]});
                }
            }
            if (a.kind == kHeld8) {
                // (past the end the code of zero)
                const uint8_t *from = (const uint8_t *)a.held + m * a.N + n;
#pragma unroll
                for (int i = 0; i < 8; ++i) code[i >> 2] |= (i < have ? (uint32_t)from[min(i, have - 1)] : 0u) << (8 * (i & 3));
                byte = a.exps[m * blocks + n / 32];
            }
            row(m, d, word, byte, z, code);          // g is zero past the end, and so is dz
        }
    }
    if (!a.sums && !a.db) return;
    if (share)
#pragma unroll
        for (int i = 0; i < 8; ++i) part[share - 1][lane][i] = sum[i];
    __syncthreads();
    if (share == 0 && have) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < kRows - 1; ++r) sum[i] += part[r][lane][i];
        if (a.db) store8((T *)a.db + n, sum, have);
        else store8(a.sums + (int64_t)blockIdx.y * a.N + n, sum, have);
    }
}

// The bias gradient from the groups' sums, always in the same order: 32 columns a workgroup, eight threads a column
// (32 groups of 8192 columns: 5 us, the latency of a launch and four loads; a thread a column took 60).
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
