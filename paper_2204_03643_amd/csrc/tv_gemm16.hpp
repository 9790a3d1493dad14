// Matrix products on bf16 operands whose rows lie on 16-byte boundaries: tiles go from memory to LDS without passing
// through registers, two buffers in turn, 32 x 32 x 16 matrix instructions.
#pragma once
#include "tv_gemm.hpp"

namespace tvl {

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __attribute__((aligned(16))) uint32_t zeros16[4];       // what a lane beyond the contraction's end loads

// Where a tile's operand comes from.  ROWS output indices (m or n) by 64 contraction indices.
//
// k contiguous: LDS holds 128 bytes a row; the 16-byte piece c of row r lies in slot c ^ ((r / 2) % 8), so that sixteen rows
// read at one c touch all 64 banks once.  Lane l of a wave's load fills slot l % 8 of the l / 8-th of eight rows.
//
// transposed (the output index contiguous): LDS holds ROWS values of one k after those of the next, as in memory; the
// transposing LDS read hands each lane four k of its column.  A read takes 64 bytes of four rows k % 4 (and of four more,
// eight further on, in the second half of the wave): 64-byte piece p of row k lies in slot p ^ (k % 4).
template <int ROWS, int WAVES, bool TRANSPOSED> struct Tile16 {
    static constexpr int kLoads = ROWS * 128 / 1024 / WAVES;       // 1024 bytes a load of a wave
    static constexpr int kPieces = ROWS / 8;                       // 16-byte pieces of one k (transposed)
    uint32_t off[kLoads];        // bytes from the tile's origin in memory
    int32_t  k[kLoads];          // contraction index of the lane's piece within a tile

    // rows: how many output indices there are from the tile's origin on (at least one)
    __device__ __forceinline__ void setup(uint32_t ld, int rows, int wave, int lane)
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int at = (j * WAVES + wave) * 64 + lane;         // 16-byte slot of the tile
            if constexpr (!TRANSPOSED) {
                const int r = at / 8, c = (at % 8) ^ ((r >> 1) & 7);
                k[j] = c * 8;
                off[j] = ((uint32_t)min(r, rows - 1) * ld + (uint32_t)c * 8) * 2;
            } else {
                const int kk = at / kPieces, c = (at % kPieces) ^ ((kk & 3) << 2);
                k[j] = kk;
                off[j] = ((uint32_t)kk * ld + (c * 8 < rows ? (uint32_t)c * 8 : 0u)) * 2;
            }
        }
    }
    // left: contraction indices that are left from the tile's origin on.  A lane beyond them loads zeros.
    template <bool WHOLE>
    __device__ __forceinline__ void load(const char *origin, char *lds, int left, int wave) const
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const char *from = origin + off[j];
            if constexpr (!WHOLE) from = k[j] < left ? from : (const char *)zeros16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(lds + (j * WAVES + wave) * 1024), 16, 0, 0);
        }
    }
    // 32 output indices from `row` on, contraction indices 16 q .. 16 q + 15: lane l has index l % 32 and k from
    // 16 q + 8 (l / 32) on.
    __device__ __forceinline__ static bf16x8 read(const char *lds, int row, int q, int lane)
    {
        if constexpr (!TRANSPOSED) {
            const int r = row + (lane & 31), c = q * 2 + (lane >> 5);
            return *(const bf16x8 *)(lds + r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
        } else {
            const int kk = q * 16 + (lane >> 5) * 8 + ((lane >> 2) & 3);
            const int col = row + (lane & 16) + (lane & 3) * 4;    // this lane's four columns of row kk
            const char *p = lds + kk * (ROWS * 2) + (((col >> 3) ^ ((kk & 3) << 2)) << 4) + (col & 4) * 2;
            typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * ROWS * 2));
            typedef int16_t s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn; each XCD takes a run of consecutive tiles, and
// consecutive tiles form columns of eight, so that what an XCD works on at a time shares rows of both operands in its L2.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tm, uint32_t tn, uint32_t &m, uint32_t &n)
{
    const uint32_t count = tm * tn, each = count / 8, more = count % 8, xcd = id % 8;
    const uint32_t t = xcd * each + min(xcd, more) + id / 8;
    const uint32_t group = t / (8 * tn), first = group * 8, rows = min(8u, tm - first);
    const uint32_t in = t - group * 8 * tn;
    m = first + in % rows;
    n = in / rows;
}

// BM x BN outputs a workgroup of WM x WN waves.
template <int BM, int BN, int WM, int WN, bool AT, bool BT>
__global__ __launch_bounds__(WM * WN * 64) void gemm16_kernel(Product g, Epilogue e)
{
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kA = BM * 128, kB = BN * 128, kOut = W / 2 * 32 * kOutPitch * 4;
    static_assert(TN == 2, "a wave's outputs are 64 columns wide");
    static_assert(kOut <= kA + kB, "the outputs' pieces fit a buffer");
    __shared__ __attribute__((aligned(1024))) char even[kA + kB];
    __shared__ __attribute__((aligned(1024))) char odd[kA + kB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int m0 = (int)tm * BM, n0 = (int)tn * BN;
    const int k0 = (int)blockIdx.y * g.k_per, k_end = min(g.K, k0 + g.k_per);
    const int steps = (k_end - k0 + 63) / 64;
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);

    Tile16<BM, W, AT> ta;
    Tile16<BN, W, BT> tb;
    ta.setup((uint32_t)g.lda, g.M - m0, wave, lane);
    tb.setup((uint32_t)g.ldb, g.N - n0, wave, lane);
    const char *pa = (const char *)g.a + (AT ? (int64_t)k0 * g.lda + m0 : (int64_t)m0 * g.lda + k0) * 2;
    const char *pb = (const char *)g.b + (BT ? (int64_t)k0 * g.ldb + n0 : (int64_t)n0 * g.ldb + k0) * 2;
    const int64_t step_a = AT ? g.lda * 128 : 128, step_b = BT ? g.ldb * 128 : 128;

    f32x16 acc[TN][TM];
#pragma unroll
    for (int i = 0; i < TN; ++i)
#pragma unroll
        for (int j = 0; j < TM; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;

    auto issue = [&](int s, char *to) {
        const int left = k_end - k0 - s * 64;
        if (left >= 64) {
            ta.template load<true>(pa, to, left, wave);
            tb.template load<true>(pb, to + kA, left, wave);
        } else {
            ta.template load<false>(pa, to, left, wave);
            tb.template load<false>(pb, to + kA, left, wave);
        }
        pa += step_a;
        pb += step_b;
    };
    auto compute = [&](const char *from) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            bf16x8 fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TN; ++i) fb[i] = Tile16<BN, W, BT>::read(from + kA, wn + 32 * i, q, lane);
#pragma unroll
            for (int j = 0; j < TM; ++j) fa[j] = Tile16<BM, W, AT>::read(from, wm + 32 * j, q, lane);
#pragma unroll
            for (int j = 0; j < TM; ++j)
#pragma unroll
                for (int i = 0; i < TN; ++i)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[i], fa[j], acc[i][j], 0, 0, 0);
        }
    };
    // a buffer's loads have landed, and nobody reads the other buffer any more
    auto turn = [&] {
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0)
        __syncthreads();
    };

    // two steps a turn of the loop, one a buffer; past the end a step of zeros
    issue(0, even);
    for (int s = 0; s < steps; s += 2) {
        turn();
        issue(s + 1, odd);
        compute(even);
        turn();
        if (s + 2 < steps) issue(s + 2, even);
        compute(odd);
    }
    __syncthreads();
    float *piece = (float *)(wave & 1 ? odd : even) + (wave >> 1) * 32 * kOutPitch;
#pragma unroll 1
    for (int j = 0; j < TM; ++j) {                    // one copy of the epilogue's code, and of its registers
#pragma unroll
        for (int jj = 0; jj < TM; ++jj)
            if (j == jj)
#pragma unroll
                for (int i = 0; i < TN; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *(f32x4 *)(piece + (lane & 31) * kOutPitch + 32 * i + q * 8 + (lane >> 5) * 4) =
                            f32x4{acc[i][jj][4 * q], acc[i][jj][4 * q + 1], acc[i][jj][4 * q + 2], acc[i][jj][4 * q + 3]};
        wave_sync();
        store_rows<bf16, 32>(piece, g, e, m0 + wm + 32 * j, n0 + wn, lane);
        wave_sync();
    }
}

}  // namespace tvl
