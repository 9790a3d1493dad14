// Matrix products of channel mixing: D[m, n] = sum_k A(m, k) B(n, k), either operand stored with k contiguous or with
// its other index contiguous (the gradients read their operands that way round), sums in 32 bits.
#pragma once
#include "tv_linear.hpp"

namespace tvl {

struct Product {
    const void *a, *b;       // A(m, k) = a[m * lda + k], or a[k * lda + m] where A is transposed; B alike
    int64_t  lda, ldb;
    int32_t  M, N, K;
    int32_t  k_per;          // contraction indices of one split, a multiple of 64
    int32_t  splits;
    float   *partial;        // [splits, M, ceil(N / 8) * 8] sums, where splits > 1
    uint32_t tiles_m, tiles_n;
};

// One 16 x 16 tile step on 16 bytes a lane of either operand: lane l holds row l % 16 of its operand and the bytes
// 16 * (l / 16) .. of 64 contraction bytes.  D's rows run over the first operand, its columns over the second: lane l
// has column l % 16, rows 4 * (l / 16) ...  In f32 four steps of four contraction indices each take one element of
// every lane's four, the same one on both sides.
template <class T> __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (sizeof(T) == 2)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
}

typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));

// 16 bytes from any address that suits T, or the first `have` elements and zeros.
template <class T> __device__ __forceinline__ u32x4 load16(const T *p, int have)
{
    constexpr int E = Elems<T>::kPer16;
    if (have >= E) {
        if constexpr (sizeof(T) == 4) return *(const u32x4_at4 *)p;
        else return *(const u32x4_at2 *)p;
    }
    u32x4 v = {0, 0, 0, 0};
    if (have <= 0) return v;
    // (every load from an element that exists, so that none of them waits for a branch)
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const uint32_t w = __float_as_uint(p[min(i, have - 1)]);
            v[i] = i < have ? w : 0u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const uint32_t w = ((const uint16_t *)p)[min(i, have - 1)];
            v[i >> 1] |= (i < have ? w : 0u) << (16 * (i & 1));
        }
    }
    return v;
}

// A wave's outputs leave through its own piece of LDS, R rows of 64 columns at a time, so that eight lanes write a
// row's 64 columns side by side (straight from the accumulators every store would touch 16 or 32 rows).  The piece's
// rows are 68 floats apart: sixteen rows of one column group then lie in different banks.
constexpr int kOutPitch = 68;

__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// PLAIN: the epilogue only rounds (the gradients' products).
template <class T, int R, bool PLAIN>
__device__ __forceinline__ void store_rows(const float *piece, const Product &g, const Epilogue &e, int m0, int n0, int lane)
{
    const int n = n0 + (lane & 7) * 8;
    const float *from = piece + (lane >> 3) * kOutPitch + (lane & 7) * 8;
    if (g.splits > 1) {
        const int64_t pitch = (g.N + 7) & ~7;
        float *to = g.partial + ((int64_t)blockIdx.y * g.M + m0 + (lane >> 3)) * pitch + n;
#pragma unroll
        for (int i = 0; i < R / 8; ++i)
            if (m0 + i * 8 + (lane >> 3) < g.M && n < g.N) {
                *(f32x4 *)(to + i * 8 * pitch) = *(const f32x4 *)(from + i * 8 * kOutPitch);
                *(f32x4 *)(to + i * 8 * pitch + 4) = *(const f32x4 *)(from + i * 8 * kOutPitch + 4);
            }
        return;
    }
    if (PLAIN && e.vec && m0 + R <= g.M && n0 + 64 <= g.N) {
        T *to = (T *)e.y + (int64_t)(m0 + (lane >> 3)) * e.ldy + n;
#pragma unroll
        for (int i = 0; i < R / 8; ++i) {
            const f32x4 a = *(const f32x4 *)(from + i * 8 * kOutPitch), b = *(const f32x4 *)(from + i * 8 * kOutPitch + 4);
            const float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            store8(to + i * 8 * e.ldy, p, 8, true);
        }
        return;
    }
#pragma unroll 1
    for (int i = 0; i < R / 8; ++i) {
        const int64_t m = m0 + i * 8 + (lane >> 3);
        const f32x4 a = *(const f32x4 *)(from + i * 8 * kOutPitch), b = *(const f32x4 *)(from + i * 8 * kOutPitch + 4);
        float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        finish8<T>(p, m, n, g.N, m < g.M, e);
    }
}

// The sums of all splits, in order, through the epilogue: eight columns a thread, four threads a block of 32.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(Product g, Epilogue e)
{
    const int per_row = (g.N + 31) / 32 * 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = at / per_row;
    const int n = (int)(at - m * per_row) * 8;
    const int64_t pitch = (g.N + 7) & ~7;
    f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
    if (m < g.M && n < g.N)
        for (int s = 0; s < g.splits; ++s) {
            const float *from = g.partial + ((int64_t)s * g.M + m) * pitch + n;
            a += *(const f32x4 *)from;
            b += *(const f32x4 *)(from + 4);
        }
    float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    finish8<T>(p, m, n, g.N, m < g.M, e);
}

}  // namespace tvl
