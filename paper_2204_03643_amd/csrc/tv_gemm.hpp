// Matrix products of channel mixing: D[m, n] = sum_k A(m, k) B(n, k), either operand stored with k contiguous or with
// its other index contiguous (the gradients read their operands that way round), sums in 32 bits.
#pragma once
#include "tv_linear.hpp"
#include <type_traits>

namespace tvl {

// f(0) .. f(N - 1), each with a constant of its own.
template <int N, int I = 0, class F> __device__ __forceinline__ void each(F f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

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

// 16 bytes from any address that suits T, or the first `have` elements and zeros.
template <class T> __device__ __forceinline__ u32x4 load16(const T *p, int have)
{
    constexpr int E = Elems<T>::kPer16;
    if (have >= E) return get16(p);
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

// A wave's outputs, PIECES pieces of R rows by 64 columns: `place(x, piece)` writes piece x there, `at(x)` says where it
// belongs.  PLAIN: the epilogue only rounds (the gradients' products).  Where the residual is read, the next piece's
// is on its way while one is worked on.
template <class T, int R, int PIECES, bool PLAIN, class Place, class At>
__device__ __forceinline__ void store_wave(float *piece, const Product &g, const Epilogue &e, int lane, Place place, At at)
{
    const int row = lane >> 3, col = (lane & 7) * 8;
    const float *from = piece + row * kOutPitch + col;
    const bool whole = at(PIECES - 1).x + R <= g.M && at(PIECES - 1).y + 64 <= g.N;      // (the last piece lies furthest)
    if (g.splits > 1) {
        const int64_t pitch = (g.N + 7) & ~7;
#pragma unroll 1
        for (int x = 0; x < PIECES; ++x) {
            place(x);
            wave_sync();
            const int2 o = at(x);
            float *to = g.partial + ((int64_t)blockIdx.y * g.M + o.x + row) * pitch + o.y + col;
#pragma unroll
            for (int i = 0; i < R / 8; ++i)
                if (o.x + i * 8 + row < g.M && o.y + col < g.N) {
                    // (a tile that was moved to end with the last column may start at any)
                    put16(to + i * 8 * pitch, *(const u32x4 *)(from + i * 8 * kOutPitch));
                    put16(to + i * 8 * pitch + 4, *(const u32x4 *)(from + i * 8 * kOutPitch + 4));
                }
            wave_sync();
        }
        return;
    }
    if (!whole) {
#pragma unroll 1
        for (int x = 0; x < PIECES; ++x) {
            place(x);
            wave_sync();
            const int2 o = at(x);
#pragma unroll 1
            for (int i = 0; i < R / 8; ++i) {
                const f32x4 a = *(const f32x4 *)(from + i * 8 * kOutPitch), b = *(const f32x4 *)(from + i * 8 * kOutPitch + 4);
                float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                finish8<T>(p, o.x + i * 8 + row, o.y + col, g.N, o.x + i * 8 + row < g.M, e);
            }
            wave_sync();
        }
        return;
    }
    constexpr int kRaw = sizeof(T) / 2;
    u32x4 res[R / 8][kRaw], next[R / 8][kRaw], bias[kRaw];
    auto ask = [&](int x) __attribute__((always_inline)) {
        const int2 o = at(x);
        const T *p = (const T *)e.res + (int64_t)(o.x + row) * e.ldr + o.y + col;
#pragma unroll
        for (int i = 0; i < R / 8; ++i)
#pragma unroll
            for (int j = 0; j < kRaw; ++j) next[i][j] = get16(p + i * 8 * e.ldr + j * (16 / (int)sizeof(T)));
    };
    if (!PLAIN && e.res) ask(0);
    int column = -1;
#pragma unroll 1
    for (int x = 0; x < PIECES; ++x) {
        const int2 o = at(x);
        if (!PLAIN && e.bias && o.y != column) {
            column = o.y;
#pragma unroll
            for (int j = 0; j < kRaw; ++j) bias[j] = get16((const T *)e.bias + o.y + col + j * (16 / (int)sizeof(T)));
        }
        if (!PLAIN && e.res) {
#pragma unroll
            for (int i = 0; i < R / 8; ++i)
#pragma unroll
                for (int j = 0; j < kRaw; ++j) res[i][j] = next[i][j];
            if (x + 1 < PIECES) ask(x + 1);
        }
        place(x);
        wave_sync();
        T *to = (T *)e.y + (int64_t)(o.x + row) * e.ldy + o.y + col;
#pragma unroll
        for (int i = 0; i < R / 8; ++i) {
            const f32x4 a = *(const f32x4 *)(from + i * 8 * kOutPitch), b = *(const f32x4 *)(from + i * 8 * kOutPitch + 4);
            float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            if (!PLAIN) {
                if (e.bias) add8<T>(p, bias);
                hold8<T>(p, o.x + i * 8 + row, o.y + col, g.N, 8, e);
                act8<sizeof(T) == 2>(p, e.act);
                if (e.res) add8<T>(p, res[i]);
            }
            store8(to + i * 8 * e.ldy, p, 8);
        }
        wave_sync();
    }
}

// The sums of all splits, in order, through the epilogue: eight columns a thread, four threads a block of 32.  Small ones are
// a launch's latency (64 x 2048 of eight splits: 4.0 us), large ones the sums' bytes (2048 x 1024 of two, 16.8 MB and 8.4: 6.8 us).
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
        for (int s = 0; s < g.splits; s += 4) {       // four splits' sums on their way together
            f32x4 va[4], vb[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *from = g.partial + ((int64_t)min(s + i, g.splits - 1) * g.M + m) * pitch + n;
                va[i] = *(const f32x4 *)from;
                vb[i] = *(const f32x4 *)(from + 4);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (s + i < g.splits) { a += va[i]; b += vb[i]; }
        }
    float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    finish8<T>(p, m, n, g.N, m < g.M, e);
}

}  // namespace tvl
