// Matrix products on bf16 operands whose rows lie on 16-byte boundaries: tiles go from memory to LDS without passing
// through registers, two or four buffers in turn, 32 x 32 x 16 matrix instructions.
//
// The matrix units bound large products: 256 x 256 outputs take 1.24 us a step of 64 by matrix instructions alone (at the clock
// that a full card keeps), 1.5 us here; 8192 x 2048 -> 8192 takes 222-236 us (1.2 PFLOP/s,
// the matrix units busy for 0.68 of the cycles), its gradients, with their transposed operands, 213 and 215 us.  Smaller tiles, for products whose large ones would leave compute units idle, are bound by
// the latency of loads: 128 x 128 and 64 x 128 with four buffers have three steps on their way (4096 x 1024 -> 1024: 13.3 us;
// 128 x 2048 -> 8192: 12.3).
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
// eight further on, in the second half of the wave): 64-byte piece p of row k lies in slot p ^ (k % 4), so that the four lie
// in different banks.  (Rows of 64 values have two pieces, and two rows fill the banks: p ^ (k / 2 % 2).)
template <int ROWS, int WAVES, bool TRANSPOSED> struct Tile16 {
    static constexpr int kLoads = ROWS * 128 / 1024 / WAVES;       // 1024 bytes a load of a wave
    static constexpr int kPieces = ROWS / 8;                       // 16-byte pieces of one k (transposed)
    uint32_t off[kLoads];        // bytes from the tile's origin in memory
    int32_t  k[kLoads];          // contraction index of the lane's piece within a tile

    __device__ __forceinline__ static int swizzle(int kk) { return ROWS >= 128 ? (kk & 3) << 2 : (kk & 2) << 1; }

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
                const int kk = at / kPieces, c = (at % kPieces) ^ swizzle(kk);
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
            const char *p = lds + kk * (ROWS * 2) + (((col >> 3) ^ swizzle(kk)) << 4) + (col & 4) * 2;
            typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * ROWS * 2));
            typedef int16_t s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// Rows of `cols` values from anywhere to rows on 16-byte boundaries, zeros up to a multiple of eight: a unit of eight a thread.
// Bound by bytes: 8192 x 2047 in 12 us, 5.6 TB/s.
__global__ __launch_bounds__(256) void copy_rows_kernel(const bf16 *from, int64_t ld, bf16 *to, int cols, int64_t units)
{
    const int64_t at = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    if (at >= units) return;
    const int per = (cols + 7) / 8;
    const int64_t row = at / per;
    const int col = (int)(at - row * per) * 8;
    *(u32x4 *)(to + at * 8) = load16(from + row * ld + col, cols - col);
}

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

// Waits until at most N of this wave's loads are on their way and its LDS reads have ended, then for all waves.
template <int N> __device__ __forceinline__ void turn()
{
    static_assert(N < 64, "");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// BM x BN outputs a workgroup of WM x WN waves, BUF buffers of 64 contraction indices.
//
// The contraction goes in steps of 64, each four times 16.  While the matrix instructions of one sixteen run, the LDS
// reads of the next are on their way; the barrier that hands a step's buffer over stands in the middle of the
// matrix instructions of its last sixteen, whose operands are in registers by then, so that the first reads of the next step
// and the loads into the freed buffer start behind running matrix instructions too.
template <int BM, int BN, int WM, int WN, int BUF, bool AT, bool BT>
__global__ __launch_bounds__(WM * WN * 64) void gemm16_kernel(Product g, Epilogue e)
{
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kA = BM * 128, kB = BN * 128, kOut = W * 32 * kOutPitch * 4;
    static_assert(TN % 2 == 0, "a wave's outputs leave 64 columns at a time");
    static_assert(kOut <= BUF * (kA + kB), "the outputs' pieces fit");
    __shared__ __attribute__((aligned(1024))) char lds[BUF][kA + kB];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int m0 = (int)tm * BM, n0 = (int)tn * BN;
    const int k0 = (int)blockIdx.y * g.k_per, k_end = min(g.K, k0 + g.k_per);
    const int steps = (k_end - k0 + 63) / 64, whole = (k_end - k0) / 64;
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);

    using TileA = Tile16<BM, W, AT>;
    using TileB = Tile16<BN, W, BT>;
    constexpr int kLoads = TileA::kLoads + TileB::kLoads;
    TileA ta;
    TileB tb;
    ta.setup((uint32_t)g.lda, g.M - m0, wave, lane);
    tb.setup((uint32_t)g.ldb, g.N - n0, wave, lane);
    const char *pa = (const char *)g.a + (AT ? (int64_t)k0 * g.lda + m0 : (int64_t)m0 * g.lda + k0) * 2;
    const char *pb = (const char *)g.b + (BT ? (int64_t)k0 * g.ldb + n0 : (int64_t)n0 * g.ldb + k0) * 2;
    const int64_t step_a = AT ? g.lda * 128 : 128, step_b = BT ? g.ldb * 128 : 128;

    f32x16 acc[TN][TM];
    each<TN * TM>([&](auto x) __attribute__((always_inline)) { acc[x % TN][x / TN] = f32x16{}; });
    bf16x8 fa[2][TM], fb[2][TN];
#pragma unroll
    for (int j = 0; j < TM; ++j) fa[1][j] = bf16x8{};
#pragma unroll
    for (int i = 0; i < TN; ++i) fb[1][i] = bf16x8{};

    // loads of one step, in order of steps; all of it is there (WHOLE) or zeros stand for what is not
    auto issue = [&](auto all, int s, char *to) {
        constexpr bool WHOLE = decltype(all)::value;
        const int left = k_end - k0 - s * 64;
        ta.template load<WHOLE>(pa, to, left, wave);
        tb.template load<WHOLE>(pb, to + kA, left, wave);
        pa += step_a;
        pb += step_b;
    };
    auto read = [&](const char *from, int q, int set) {
#pragma unroll
        for (int i = 0; i < TN; ++i) fb[set][i] = TileB::read(from + kA, wn + 32 * i, q, lane);
#pragma unroll
        for (int j = 0; j < TM; ++j) fa[set][j] = TileA::read(from, wm + 32 * j, q, lane);
    };
    auto multiply = [&](auto set, auto first, auto last) __attribute__((always_inline)) {     // the set's matrix instructions first .. last - 1
        each<last - first>([&](auto y) __attribute__((always_inline)) {
            constexpr int x = first + y, i = x % TN, j = x / TN;
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[set][i], fa[set][j], acc[i][j], 0, 0, 0);
        });
    };
    constexpr int kAll = TM * TN, kHalf = kAll / 2;
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};
    constexpr std::integral_constant<int, kHalf> cHalf{};
    constexpr std::integral_constant<int, kAll> cAll{};
    // the order of a run of matrix instructions and of what goes behind them: the LDS reads, two after each at least, and
    // the next loads, spread over the step's first one and a half sixteens
    auto order = [&](auto count, auto with_loads) {
        constexpr int kReads = TM * (AT ? 2 : 1) + TN * (BT ? 2 : 1);
        constexpr int n = decltype(count)::value, kEach = (kReads + n - 1) / n > 2 ? (kReads + n - 1) / n : 2;
        constexpr int kLoadsEach = (kLoads + kAll + kHalf - 1) / (kAll + kHalf);
#pragma unroll
        for (int x = 0; x < n; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (x * kEach < kReads) __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);
            if constexpr (decltype(with_loads)::value) __builtin_amdgcn_sched_group_barrier(0x010, kLoadsEach, 0);
        }
    };
    // (`to` and `from` are told apart by __restrict: otherwise the compiler takes every LDS read for one of what is still
    // being loaded, and waits for all loads)
    auto step = [&](auto all, char *__restrict to, const char *__restrict from, int s) {
        read(from, 0, 0);
        multiply(c1, cHalf, cAll);
        if (decltype(all)::value || s - 1 + BUF < steps) issue(all, s - 1 + BUF, to);
        order(std::integral_constant<int, kAll - kHalf>{}, all);
        read(from, 1, 1);
        multiply(c0, c0, cAll);
        order(cAll, all);
        read(from, 2, 0);
        multiply(c1, c0, cAll);
        order(cAll, std::false_type{});
        read(from, 3, 1);
        multiply(c0, c0, cAll);
        order(cAll, std::false_type{});
        multiply(c1, c0, cHalf);
    };
#pragma unroll
    for (int s = 0; s < BUF - 1; ++s)
        if (s < whole) issue(std::true_type{}, s, lds[s]);
        else if (s < steps) issue(std::false_type{}, s, lds[s]);
    if (steps >= BUF - 1) turn<(BUF - 2) * kLoads>();
    else turn<0>();
    // step s's loads are this wave's oldest: they have landed when no more than those of the steps after it are on their
    // way; behind the barrier everybody's have, and nobody reads the buffer of step s - 1 any more
    int fill = BUF - 1, from = 0, s = 0;
    for (; s - 1 + BUF < whole; ++s) {
        step(std::true_type{}, lds[fill], lds[from], s);
        turn<(BUF - 2) * kLoads>();
        fill = from;
        from = from + 1 == BUF ? 0 : from + 1;
    }
    for (; s < steps; ++s) {
        step(std::false_type{}, lds[fill], lds[from], s);
        turn<0>();
        fill = from;
        from = from + 1 == BUF ? 0 : from + 1;
    }
    multiply(c1, cHalf, cAll);

    float *piece = (float *)lds + wave * 32 * kOutPitch;
    store_wave<bf16, 32, TM * TN / 2, AT || BT>(piece, g, e, lane,
        [&](int x) __attribute__((always_inline)) {  // (one copy of the epilogue's code, whichever the accumulators)
            each<TM * TN / 2>([&](auto y) __attribute__((always_inline)) {
                if (x == y)
                    each<2>([&](auto i) __attribute__((always_inline)) {
                        f32x16 a = acc[y / TM * 2 + i][y % TM];
                        asm volatile("" : "+v"(a));   // (or the compiler joins the branches by the accumulators' addresses)
                        each<4>([&](auto z) __attribute__((always_inline)) {
                            constexpr int q = 4 * z;
                            *(f32x4 *)(piece + (lane & 31) * kOutPitch + 32 * i + 2 * q + (lane >> 5) * 4) =
                                f32x4{a[q], a[q + 1], a[q + 2], a[q + 3]};
                        });
                    });
            });
        },
        [&](int x) __attribute__((always_inline)) { return int2{m0 + wm + x % TM * 32, n0 + wn + x / TM * 64}; });
}

}  // namespace tvl
