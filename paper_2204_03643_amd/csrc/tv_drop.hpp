// Dropout from a counter-based generator: which columns of a row are dropped is computed from (seed, offset, row, column)
// wherever it is needed, so that no mask is stored and the backward call makes the same one.
//
// Philox 4x32-10 of Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3" (2011): ten rounds of two
// 32 x 32 -> 64 bit products each.  16 bits a column: eight columns share a call, which is what a lane has of a row anyway.  The
// bytes bound the kernel: 8192 x 8192 in bf16 50 us, 5.4 TB/s, and where everything is still in the last cache 33 us with ten rounds
// or with one.
#pragma once
#include "tv_linear.hpp"

namespace tvl {

struct Drop {
    uint64_t seed, offset;
    const int64_t *seed_at;
    uint32_t below;          // a column is dropped where its number is below
    float    factor;         // of what is kept
};

struct DropKey { uint32_t k0, k1, o0, o1; };
__device__ __forceinline__ DropKey drop_key(const Drop &d)
{
    const uint64_t seed = d.seed + (d.seed_at ? (uint64_t)*d.seed_at : 0u);
    return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)d.offset, (uint32_t)(d.offset >> 32)};
}

// The eight numbers of columns 8 group .. 8 group + 7 of a row, two to a word, the lower half first.
__device__ __forceinline__ u32x4 drop_numbers(DropKey k, uint32_t row, uint32_t group)
{
    uint32_t c0 = group, c1 = row, c2 = k.o0, c3 = k.o1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k.k0;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k.k1;
        c1 = (uint32_t)p1;
        c3 = (uint32_t)p0;
        k.k0 += 0x9E3779B9u;
        k.k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

__device__ __forceinline__ bool dropped(u32x4 numbers, int i, const Drop &d)
{
    return (i & 1 ? numbers[i >> 1] >> 16 : numbers[i >> 1] & 0xffffu) < d.below;
}
// v is zero where a column is dropped, whatever it was, and the factor times as large elsewhere.
__device__ __forceinline__ void drop8(float (&v)[8], u32x4 numbers, const Drop &d)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = dropped(numbers, i, d) ? 0.0f : v[i] * d.factor;
}
// The same without the factor: for what a dropped place's gradient of 0 is multiplied by, which could be infinite or a NaN.
__device__ __forceinline__ void clear8(float (&v)[8], u32x4 numbers, const Drop &d)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = dropped(numbers, i, d) ? 0.0f : v[i];
}

// Rows of n values, `lanes` lanes (a power of two, at most 256) side by side in a row, eight values each.
template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(const T *x, T *y, int64_t rows, int n, int64_t ldx, int shift, Drop d)
{
    const DropKey key = drop_key(d);
    const int lanes = 1 << shift, per = (n + 7) / 8;
    const int64_t step = (int64_t)gridDim.x * (256 >> shift);
    for (int64_t row = (int64_t)blockIdx.x * (256 >> shift) + (threadIdx.x >> shift); row < rows; row += step)
        for (int group = threadIdx.x & (lanes - 1); group < per; group += lanes) {
            const int have = min(8, n - group * 8);
            float v[8];
            get8(v, x + row * ldx + group * 8, have);
            drop8(v, drop_numbers(key, (uint32_t)row, (uint32_t)group), d);
            store8(y + row * n + group * 8, v, have);
        }
}

}  // namespace tvl
