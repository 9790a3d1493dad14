// Products of a few rows (single tokens and small batches of them): D[m, n] = sum_k x[m, k] W[n, k], M at most 64.
//
// W is read once, straight into the matrix instructions' registers: what bounds the kernel is W's bytes, or for a small W
// the latency of one pass.  One row, 2048 -> 8192: bf16 8.1 us, 4.1 TB/s; f32 19.6 us, 3.4 TB/s; 256 -> 256 takes 4.5 us a call,
// nothing but its launch.  A workgroup of eight waves has 16 NT columns; the waves share out the contraction in turns
// of 64 bytes of every row, so that they read 512 neighbouring bytes of a row together, and their sums are joined in
// LDS, in order.  x (at most 64 rows) is read again by every workgroup, out of L2.
#pragma once
#include "tv_gemm.hpp"

namespace tvl {

// MT: tiles of 16 rows.  NT: tiles of 16 columns.  UNROLL: turns whose loads are in flight together.
template <class T, int MT, int NT, int UNROLL>
__global__ __launch_bounds__(512) void gemv_kernel(Product g, Epilogue e)
{
    constexpr int E = Elems<T>::kPer16, kTurn = 4 * E, kWaves = 8;      // contraction indices of a wave's turn
    constexpr int kPitch = NT * 16 + 4;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][MT * 16 * kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (int)blockIdx.x * (NT * 16), row = lane & 15, piece = (lane >> 4) * E;

    const T *pw[NT], *px[MT];
#pragma unroll
    for (int i = 0; i < NT; ++i) pw[i] = (const T *)g.b + (int64_t)min(n0 + 16 * i + row, g.N - 1) * g.ldb + piece;
#pragma unroll
    for (int j = 0; j < MT; ++j) px[j] = (const T *)g.a + (int64_t)min(16 * j + row, g.M - 1) * g.lda + piece;
    f32x4 acc[NT][MT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int k_first = (int)blockIdx.y * g.k_per, k_end = min(g.K, k_first + g.k_per);
    const int whole = (k_end - k_first) / kTurn;     // turns; what is left of the contraction comes last
    for (int turn = wave; turn < whole; turn += UNROLL * kWaves) {
        u32x4 fw[UNROLL][NT], fx[UNROLL][MT];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int k = k_first + (turn + u * kWaves) * kTurn;
            if (turn + u * kWaves < whole) {         // the same for all lanes
#pragma unroll
                for (int i = 0; i < NT; ++i) fw[u][i] = load16(pw[i] + k, E);
#pragma unroll
                for (int j = 0; j < MT; ++j) fx[u][j] = load16(px[j] + k, E);
            } else {
#pragma unroll
                for (int i = 0; i < NT; ++i) fw[u][i] = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < MT; ++j) fx[u][j] = u32x4{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int j = 0; j < MT; ++j) acc[i][j] = mma<T>(fw[u][i], fx[u][j], acc[i][j]);
    }
    const int k = k_first + whole * kTurn;
    if (k < k_end && whole % kWaves == wave) {
        const int have = k_end - k - piece;
        u32x4 fw[NT], fx[MT];
#pragma unroll
        for (int i = 0; i < NT; ++i) fw[i] = load16(pw[i] + k, have);
#pragma unroll
        for (int j = 0; j < MT; ++j) fx[j] = load16(px[j] + k, have);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[i][j] = mma<T>(fw[i], fx[j], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j)
            *(f32x4 *)&sums[wave][(16 * j + row) * kPitch + 16 * i + (lane >> 4) * 4] = acc[i][j];
    __syncthreads();
    // whole waves: NT * 2 threads a row, eight columns each
    for (int at = (int)threadIdx.x; at < MT * 16 * NT * 2; at += 512) {
        const int m = at / (NT * 2), c = at % (NT * 2) * 8, n = n0 + c;
        f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            a += *(const f32x4 *)&sums[w][m * kPitch + c];
            b += *(const f32x4 *)&sums[w][m * kPitch + c + 4];
        }
        if (g.splits > 1) {
            if (m < g.M && n < g.N) {
                float *to = g.partial + ((int64_t)blockIdx.y * g.M + m) * ((g.N + 7) & ~7) + n;
                *(f32x4 *)to = a;
                *(f32x4 *)(to + 4) = b;
            }
        } else {
            float p[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
            finish8<T>(p, m, n, g.N, m < g.M, e);
        }
    }
}

}  // namespace tvl
