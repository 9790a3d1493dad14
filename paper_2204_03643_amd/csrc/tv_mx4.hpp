// Values in 4 bits: blocks of 32 values of a row with a common power of two (elements e2m1, scales e8m0 of the OCP
// microscaling formats), as the matrix instructions take them: 16 bytes of codes are a lane's operand, a byte its scale.
//
// A row's codes are padded to whole groups of 128 values (64 bytes); the four scale bytes of a group make a word, and the
// words of one group of all rows lie side by side, so that the scales of a tile's rows are one contiguous read.
// Reads and writes are all there is: 2 + 1/2 + 1/32 bytes a value (bf16) each way; 16384 x 4096: 33 us (5.1 TB/s) either way.
#pragma once
#include "tv_linear.hpp"

namespace tvl {

constexpr int kGroup4 = 128;          // values of a group: four blocks

__host__ __device__ inline int64_t groups4(int64_t n) { return (n + kGroup4 - 1) / kGroup4; }
__host__ __device__ inline int64_t rows4(int64_t rows) { return (rows + 3) & ~(int64_t)3; }      // of an array of scale words

// The scale of a block from its largest magnitude's bits: 2^(e - 2), 2^e the power of two at or below it (2^-120 at least),
// so that the largest value over the scale is in [4, 8); 255 where a value is not finite.
__device__ __forceinline__ uint32_t scale4_byte(uint32_t top)
{
    return top >= 0x7f800000u ? 255u : (max(top, kLeastMagnitude) >> 23) - 2u;
}
__device__ __forceinline__ float scale4_value(uint32_t byte)
{
    return __uint_as_float(byte == 255u ? 0x7fc00000u : byte == 0u ? 0x00400000u : byte << 23);
}

// Four bytes of codes of eight values over a scale.  The conversion instruction rounds to nearest, halfway cases to the even
// code, and clamps to 6 (tried on all bf16 values and on f32 values next to the borders, with scales of 2^-122 to 2^125).
__device__ __forceinline__ uint32_t codes4_of(const float (&v)[8], float scale)
{
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    return c;
}

// 16 lanes a group of a row, eight values a lane; a workgroup has 16 rows at a time, so that their scale words leave side by
// side, and U groups, whose loads are on their way together.  Workgroups next to each other have groups next to each other
// (rows next to each other: 41 us in place of 33).
template <class T, int U>
__global__ __launch_bounds__(256) void mx4_save_kernel(const T *x, int64_t ldx, uint8_t *codes, uint32_t *exps, int64_t rows,
                                                       int n, int groups)
{
    const int lane = threadIdx.x & 15;
    const int64_t pitch = rows4(rows);
    for (int64_t row = (int64_t)blockIdx.y * 16 + (threadIdx.x >> 4); row < pitch; row += (int64_t)gridDim.y * 16)
        for (int first = blockIdx.x * U; first < groups; first += gridDim.x * U) {
            float v[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = (first + u) * kGroup4 + lane * 8;
                get8(v[u], x + row * ldx + k, row < rows && first + u < groups ? max(0, min(8, n - k)) : 0);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int g = first + u, k = g * kGroup4 + lane * 8;
                if (g >= groups) break;
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7fffffffu);
                top = max(top, (uint32_t)__shfl_xor(top, 1));
                top = max(top, (uint32_t)__shfl_xor(top, 2));
                uint32_t byte = scale4_byte(top);
                const uint32_t c = byte == 255u ? 0u : codes4_of(v[u], __uint_as_float(byte << 23));
                if ((k & ~31) >= n || row >= rows) byte = 127u;          // a block that only fills up
                byte <<= 8 * (lane >> 2);
                byte |= (uint32_t)__shfl_xor(byte, 4);
                byte |= (uint32_t)__shfl_xor(byte, 8);
                if (row < rows) *(uint32_t *)(codes + row * groups * 64 + g * 64 + lane * 4) = c;
                if (lane == 0) exps[g * pitch + row] = byte;
            }
        }
}

template <class T>
__global__ __launch_bounds__(256) void mx4_load_kernel(const uint8_t *codes, const uint8_t *exps, T *x, int64_t ldx, int64_t rows,
                                                       int n, int groups)
{
    const int lane = threadIdx.x & 15;
    const int64_t pitch = rows4(rows);
    for (int64_t row = (int64_t)blockIdx.y * 16 + (threadIdx.x >> 4); row < rows; row += (int64_t)gridDim.y * 16)
        for (int g = blockIdx.x; g < groups; g += gridDim.x) {
            const int k = g * kGroup4 + lane * 8, have = max(0, min(8, n - k));
            if (have == 0) continue;
            const uint32_t c = *(const uint32_t *)(codes + row * groups * 64 + g * 64 + lane * 4);
            const float scale = scale4_value(exps[(g * pitch + row) * 4 + (lane >> 2)]);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // sign, two bits of exponent, one of fraction: 0 and 1/2 below the smallest exponent
                const uint32_t q = c >> (4 * i), e = (q >> 1) & 3u, f = q & 1u;
                const float a = e ? __uint_as_float((126u + e) << 23 | f << 22) : 0.5f * (float)f;
                v[i] = __uint_as_float(__float_as_uint(a) | (q & 8u) << 28) * scale;
            }
            store8(x + row * ldx + k, v, have);
        }
}

}  // namespace tvl
