// 8-bit activation checkpoints: a [rows, n] tensor as a code a sample and a step byte a block of 32 samples of a row.
//
// Reads and writes are all there is: 2 + 1 + 1/32 bytes a sample (bf16) each way.
#pragma once
#include "tv_linear.hpp"

namespace tvl {

// Four lanes a block, eight consecutive samples a lane; the block's magnitude is the largest of the four lanes'.
template <class T>
__global__ __launch_bounds__(256) void ckpt8_save_kernel(const T *x, int64_t ldx, int8_t *codes, uint8_t *exps,
                                                         int64_t rows, int n, int blocks, uint32_t vec)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 64 + (threadIdx.x >> 2);
    const int64_t row = at / blocks;
    if (row >= rows) return;                     // whole groups of four lanes
    const int block = (int)(at - row * blocks), lane = threadIdx.x & 3;
    const int k = block * kBlock + lane * 8, have = max(0, min(8, n - k));
    const T *from = x + row * ldx + k;
    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (have == 8 && vec) {
        const f32x4 a = load4(from, 4, true), b = load4(from + 4, 4, true);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) v[i] = widen(from[i]);
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[i]));
    top = max(top, (uint32_t)__shfl_xor(top, 1));
    top = max(top, (uint32_t)__shfl_xor(top, 2));
    const uint32_t byte = step_byte(top);
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i >> 2] |= ((uint32_t)code_of(v[i], byte) & 255u) << (8 * (i & 3));
    if (lane == 0) exps[at] = (uint8_t)byte;
    int8_t *to = codes + row * n + k;
    if (have == 8 && vec) *(u32x2 *)to = u32x2{c[0], c[1]};
    else
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) to[i] = (int8_t)(c[i >> 2] >> (8 * (i & 3)));
}

template <class T>
__global__ __launch_bounds__(256) void ckpt8_load_kernel(const int8_t *codes, const uint8_t *exps, T *x, int64_t ldx,
                                                         int64_t rows, int n, int blocks, uint32_t vec)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 64 + (threadIdx.x >> 2);
    const int64_t row = at / blocks;
    if (row >= rows) return;
    const int block = (int)(at - row * blocks), lane = threadIdx.x & 3;
    const int k = block * kBlock + lane * 8, have = max(0, min(8, n - k));
    if (have == 0) return;
    const uint32_t byte = exps[at];
    const int8_t *from = codes + row * n + k;
    T *to = x + row * ldx + k;
    if (have == 8 && vec) {
        const u32x2 c = *(const u32x2 *)from;
        f32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = value_of((int)(int8_t)(c[0] >> (8 * i)), byte);
            b[i] = value_of((int)(int8_t)(c[1] >> (8 * i)), byte);
        }
        store4(to, a, 4, true);
        store4(to + 4, b, 4, true);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) to[i] = narrow<T>(value_of(from[i], byte));
    }
}

}  // namespace tvl
