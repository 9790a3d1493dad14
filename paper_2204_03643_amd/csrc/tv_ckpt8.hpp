// 8-bit activation checkpoints: a [rows, n] tensor as a code a sample and a step byte a block of 32 samples of a row.
//
// Reads and writes are all there is: 2 + 1 + 1/32 bytes a sample (bf16) each way.  8192 x 8192 in bf16: 43 us to save, 49
// to restore (4.7 and 4.2 TB/s).
#pragma once
#include "tv_linear.hpp"

namespace tvl {

// Four lanes a block, eight consecutive samples a lane; the block's magnitude is the largest of the four lanes'.
template <class T>
__global__ __launch_bounds__(256) void ckpt8_save_kernel(const T *x, int64_t ldx, int8_t *codes, uint8_t *exps,
                                                         int64_t rows, int n, int blocks)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 64 + (threadIdx.x >> 2);
    const int64_t row = at / blocks;
    if (row >= rows) return;                     // whole groups of four lanes
    const int block = (int)(at - row * blocks), lane = threadIdx.x & 3;
    const int k = block * kBlock + lane * 8, have = max(0, min(8, n - k));
    float v[8];
    load8(v, x + row * ldx + k, have);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, finite_magnitude(v[i]));
    top = max(top, (uint32_t)__shfl_xor(top, 1));
    top = max(top, (uint32_t)__shfl_xor(top, 2));
    const uint32_t byte = step_byte(top);
    u32x2 c = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i >> 2] |= ((uint32_t)code_of(v[i], byte) & 255u) << (8 * (i & 3));
    if (lane == 0) exps[at] = (uint8_t)byte;
    store_codes(codes + row * n + k, c, have);
}

template <class T>
__global__ __launch_bounds__(256) void ckpt8_load_kernel(const int8_t *codes, const uint8_t *exps, T *x, int64_t ldx,
                                                         int64_t rows, int n, int blocks)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 64 + (threadIdx.x >> 2);
    const int64_t row = at / blocks;
    if (row >= rows) return;
    const int block = (int)(at - row * blocks), lane = threadIdx.x & 3;
    const int k = block * kBlock + lane * 8, have = max(0, min(8, n - k));
    if (have == 0) return;
    const uint32_t byte = exps[at];
    const int8_t *from = codes + row * n + k;
    float v[8];
    if (have == 8) {
        const u32x2 c = *(const u32x2_at1 *)from;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = value_of((int)(int8_t)(c[i >> 2] >> (8 * (i & 3))), byte);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = value_of(from[min(i, have - 1)], byte);
    }
    store8(x + row * ldx + k, v, have);
}

}  // namespace tvl
