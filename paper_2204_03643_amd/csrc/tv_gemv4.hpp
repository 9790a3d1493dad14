// Products of a few rows with a weight in 4 bits: D[m, n] = sum_k X(m, k) W(n, k), M at most 32.
//
// W is read once, straight into the matrix instructions' registers (16 x 16 x 128: a lane has a block of 32 of one row):
// what bounds the kernel is W's bytes, or for a small W the latency of one pass.  A workgroup of eight waves has 16, 32 or 64
// columns (where there are many: what it makes of x, five times the loads of 16 columns' weight and about eighty vector instructions
// a group, serves them all); the waves share out the groups of 128 in turn, so that they read 512 neighbouring bytes of a row together, and
// their sums are joined in LDS, in order.  One row, x taken to 4 bits included, in a graph: 2048 -> 8192 5.1 us, 4096 -> 16384
// 8.7 (W's 35.7 MB in 7.1 at the rate of a copy).
#pragma once
#include "tv_gemm4.hpp"

namespace tvl {

// x as it comes (OWN: rows of T, which every workgroup takes to 4 bits by itself: a lane has a whole block, so that its scale
// needs no other lane) or as codes.
struct Rows4 {
    const void *p;
    const uint32_t *scales;
    int64_t ld;              // OWN
    uint32_t rows;           // of a group's scale words
    int32_t K;               // values of a row (OWN)
};

struct Piece4 {
    u32x4 codes;
    int   scale;
};

template <class T, bool OWN> struct RawPiece4 {
    u32x4 raw[OWN ? 2 * sizeof(T) : 1];
    int   scale;

    __device__ __forceinline__ void load(const Rows4 &x, int row, int group, int block, int64_t pitch)
    {
        if constexpr (OWN) {
            const T *p = (const T *)x.p + (int64_t)row * x.ld + group * kGroup4 + block * 32;
            const int have = x.K - group * kGroup4 - block * 32;
            constexpr int E = Elems<T>::kPer16;
#pragma unroll
            for (int i = 0; i < (int)(2 * sizeof(T)); ++i) raw[i] = load16(p + i * E, have - i * E);
        } else {
            raw[0] = *(const u32x4 *)((const char *)x.p + ((int64_t)row * pitch + group) * 64 + block * 16);
            scale = (int)(x.scales[(int64_t)group * x.rows + row] >> (8 * block));
        }
    }
    __device__ __forceinline__ Piece4 get() const
    {
        if constexpr (!OWN) return {raw[0], scale};
        else {
            uint32_t top = 0;
            if constexpr (sizeof(T) == 2) {          // the largest of two at a time, as they lie
                typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
                u16x2 most = {0, 0};
#pragma unroll
                for (int i = 0; i < 16; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, raw[i >> 2][i & 3] & 0x7fff7fffu));
                top = (uint32_t)max(most[0], most[1]) << 16;
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) top = max(top, raw[i >> 2][i & 3] & 0x7fffffffu);
            }
            const uint32_t byte = scale4_byte(top);
            Piece4 o{{0, 0, 0, 0}, (int)byte};
            if (byte != 255u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (sizeof(T) == 2) v[j] = __uint_as_float(j & 1 ? raw[i][j >> 1] & 0xffff0000u : raw[i][j >> 1] << 16);
                        else v[j] = __uint_as_float(raw[2 * i + (j >> 2)][j & 3]);
                    }
                    o.codes[i] = codes4_of(v, __uint_as_float(byte << 23));
                }
            return o;
        }
    }
};

// MT: tiles of 16 rows.  NT: tiles of 16 columns, which share what is made of x.  UNROLL: groups whose loads are in flight
// together.
template <class T, int MT, int NT, int UNROLL, bool OWN>
__global__ __launch_bounds__(512) void gemv4_kernel(Product g, Rows4 x, const uint32_t *w_scales, uint32_t w_rows, Epilogue e)
{
    constexpr int kWaves = 8, kPitch = NT * 16 + 4, kFinish = MT * 16 * NT * 2;      // two threads a row and tile finish it
    static_assert(kFinish <= 512, "eight columns a thread");
    __shared__ __attribute__((aligned(16))) float sums[kWaves][MT * 16 * kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (int)blockIdx.x * (NT * 16), row = lane & 15, block = lane >> 4;
    const int64_t pitch = g.ldb / 32;                // groups of a row
    const char *pw[NT];
    const uint32_t *ps[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int n = min(n0 + 16 * i + row, g.N - 1);
        pw[i] = (const char *)g.b + (int64_t)n * pitch * 64 + block * 16;
        ps[i] = w_scales + n;
    }
    // bias and residual are on their way before anything else
    const int m = threadIdx.x / (NT * 2), column = n0 + threadIdx.x % (NT * 2) * 8;
    const int have = m < min(MT * 16, g.M) ? max(0, min(8, g.N - column)) : 0;
    float bias[8], res[8];
    if (e.bias) load8(bias, (const T *)e.bias + column, have);
    if (e.res) load8(res, (const T *)e.res + (int64_t)m * e.ldr + column, have);
    f32x4 acc[NT][MT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int end = g.K / 32;
    for (int k = wave; k < end; k += UNROLL * kWaves) {
        u32x4 fw[UNROLL][NT];
        uint32_t sw[UNROLL][NT];
        RawPiece4<T, OWN> fx[UNROLL][MT];
        // (beyond the end the last group once more: what is loaded is not multiplied)
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int at = min(k + u * kWaves, end - 1);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                fw[u][i] = *(const u32x4 *)(pw[i] + (int64_t)at * 64);
                sw[u][i] = ps[i][(int64_t)at * w_rows];
            }
#pragma unroll
            for (int j = 0; j < MT; ++j) fx[u][j].load(x, min(16 * j + row, g.M - 1), at, block, pitch);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (k + u * kWaves >= end) break;        // the same for all lanes
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const Piece4 p = fx[u][j].get();
#pragma unroll
                for (int i = 0; i < NT; ++i)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand4(fw[u][i]), operand4(p.codes), acc[i][j], 4, 4, 0,
                                                                                 (int)(sw[u][i] >> (8 * block)), 0, p.scale);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) *(f32x4 *)&sums[wave][(16 * j + row) * kPitch + 16 * i + block * 4] = acc[i][j];
    __syncthreads();
    if (have) {
        const float *from = sums[0] + m * kPitch + threadIdx.x % (NT * 2) * 8;
        f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            a += *(const f32x4 *)(from + w * (MT * 16 * kPitch));
            b += *(const f32x4 *)(from + w * (MT * 16 * kPitch) + 4);
        }
        float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        if (e.bias)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] += bias[i];
        act8<sizeof(T) == 2>(p, e.act);
        if (e.res)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] += res[i];
        store8((T *)e.y + (int64_t)m * e.ldy + column, p, have);
    }
}

}  // namespace tvl
