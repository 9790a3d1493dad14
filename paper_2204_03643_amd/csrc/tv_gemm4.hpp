// Products of values in 4 bits on tiles: D[m, n] = sum_k X(m, k) W(n, k), both in blocks of 32 with a scale each.
//
// A block's 16 bytes of codes are what a lane hands to a scaled matrix instruction (32 x 32 x 64).  Tiles go from memory to
// LDS without passing through registers; the scales come beside them, a word of four for each group of 128, and a lane picks
// those of its blocks with one permutation a step.
//
// 256 x 256 outputs take 1.75 us a step of 256 on a full card, 4.6 PFLOP/s (the matrix instructions alone reach 8.2): the tiles'
// bytes come out of L2 at 10 TB/s, whose channels are busy for 0.70 of the cycles, the matrix units for 0.55, at the 1.8 GHz that a full
// card keeps (64 workgroups on an otherwise idle card: 0.77 us a step).  Smaller tiles read more: 128 x 256 on two workgroups
// a compute unit, whose epilogues run behind each other's products, took 305 us for 8192 x 8192 -> 8192 in place of 257, and 98
// in place of 92 for 8192 x 2048 -> 8192.  Of those 92, 26 are the outputs' bytes; gelu adds 28, and outputs in f32 24 (with
// gelu 63).  Four waves of 128 x 128, four buffers of
// half a step and streaming stores changed times by -3 to +5 %.
#pragma once
#include "tv_gemm16.hpp"
#include "tv_mx4.hpp"

namespace tvl {

typedef int32_t s32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ s32x8 operand4(u32x4 v)
{
    return s32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}

// Scale words of x and W; a group of all rows lies together, `rows` (a multiple of four) words.
struct Scales {
    const uint32_t *x, *w;
    uint32_t x_rows, w_rows;
};

// The codes of ROWS rows by G groups a step.  LDS holds 64 G bytes a row; the 16-byte block c of row r lies in slot
// c ^ (r / 2) % 8 (two groups) or c ^ (r / 4) % 4 (one), so that sixteen rows read at one c touch all 64 banks once.
template <int ROWS, int WAVES, int G> struct Tile4 {
    static constexpr int kBlocks = 4 * G, kLoads = ROWS * kBlocks / 64 / WAVES;      // 1024 bytes a load of a wave
    uint32_t off[kLoads];        // bytes from the tile's origin in memory
    int32_t  group[kLoads];      // of the lane's block within a step

    __device__ __forceinline__ static int swizzle(int r) { return G == 2 ? (r >> 1) & 7 : (r >> 2) & 3; }

    // pitch: bytes of a row; rows: how many there are from the tile's origin on (at least one)
    __device__ __forceinline__ void setup(uint32_t pitch, int rows, int wave, int lane)
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int at = (j * WAVES + wave) * 64 + lane, r = at / kBlocks, c = at % kBlocks ^ swizzle(r);
            group[j] = c / 4;
            off[j] = (uint32_t)min(r, rows - 1) * pitch + (uint32_t)c * 16;
        }
    }
    // groups: how many are left from the step on.  A lane beyond them loads zeros.
    template <bool WHOLE>
    __device__ __forceinline__ void load(const char *origin, char *lds, int groups, int wave) const
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const char *from = origin + off[j];
            if constexpr (!WHOLE) from = group[j] < groups ? from : (const char *)zeros16;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                             (__attribute__((address_space(3))) void *)(lds + (j * WAVES + wave) * 1024), 16, 0, 0);
        }
    }
    // 32 rows from `row` on, blocks 2 q and 2 q + 1: lane l has row l % 32 and block 2 q + l / 32.
    __device__ __forceinline__ static u32x4 read(const char *lds, int row, int q, int lane)
    {
        const int r = row + (lane & 31), c = q * 2 + (lane >> 5);
        return *(const u32x4 *)(lds + r * (64 * G) + ((c ^ swizzle(r)) << 4));
    }
};

// The scale words of a tile's step, in pieces of 256 words: those of 256 rows and a group, or of fewer rows and both groups
// (what is left of a piece repeats its beginning).  A wave loads one piece; where there are more waves than pieces some load the
// same one to the same place, so that all waves have as many loads on their way.
template <int BM, int BN, int G> struct Scales4 {
    static constexpr int kX = BM == 256 ? G : 1, kW = BN == 256 ? G : 1, kPieces = kX + kW;
    const char *from;
    int64_t step;            // bytes to the next step
    uint32_t back;           // bytes from the lane's words of a step's second group to those of its first; 0 in the first
    int32_t piece;

    __device__ __forceinline__ void setup(const Scales &s, uint32_t m0, uint32_t n0, int first, int wave, int lane)
    {
        piece = wave % kPieces;
        const bool of_x = piece < kX;
        const uint32_t rows = of_x ? BM : BN, pitch = of_x ? s.x_rows : s.w_rows, at = (uint32_t)lane * 4;
        const uint32_t group = rows == 256 ? (uint32_t)(of_x ? piece : piece - kX) : at / rows % G;
        const uint32_t row = min((of_x ? m0 : n0) + at % rows, pitch - 4);
        from = (const char *)((of_x ? s.x : s.w) + ((int64_t)first + group) * pitch + row);
        step = (int64_t)pitch * 4 * G;
        back = group ? pitch * 4 : 0;
    }
    __device__ __forceinline__ void load(char *lds, int groups)
    {
        const char *p = G == 1 || groups >= G ? from : from - back;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p,
                                         (__attribute__((address_space(3))) void *)(lds + piece * 1024), 16, 0, 0);
        from += step;
    }
    // The scales of 32 rows from `row` on: lane l has those of row l % 32, byte q that of block 2 q + l / 32 of the step.
    template <int ROWS> __device__ __forceinline__ static uint32_t read(const char *words, int row, int lane)
    {
        const uint32_t *w = (const uint32_t *)words + row + (lane & 31);
        return __builtin_amdgcn_perm(w[G == 2 ? ROWS : 0], w[0], lane < 32 ? 0x06040200u : 0x07050301u);
    }
};

// BM x BN outputs a workgroup of WM x WN waves, BUF buffers of G groups.  g counts codes by twos of bytes: lda, ldb and K are
// 32 a group.
//
// The order of things is that of the products in 16 bits: while the matrix instructions of one pair of blocks run, the LDS
// reads of the next are on their way, and the barrier that hands a step's buffer over stands in the middle of the matrix
// instructions of its last pair, whose operands are in registers by then.
template <class T, int BM, int BN, int WM, int WN, int BUF, int G>
__global__ __launch_bounds__(WM * WN * 64) void gemm4_kernel(Product g, Scales scales, Epilogue e)
{
    using S = Scales4<BM, BN, G>;
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32, kStep = 32 * G, kPairs = 2 * G;
    constexpr int kA = BM * 64 * G, kB = BN * 64 * G, kS = S::kPieces * 1024, kOut = W * 32 * kOutPitch * 4;
    static_assert(TN % 2 == 0, "a wave's outputs leave 64 columns at a time");
    static_assert(W >= S::kPieces, "the waves load all scales");
    static_assert(kOut <= BUF * (kA + kB + kS), "the outputs' pieces fit");
    __shared__ __attribute__((aligned(1024))) char lds[BUF][kA + kB + kS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int m0 = (int)tm * BM, n0 = (int)tn * BN;
    const int k0 = (int)blockIdx.y * g.k_per, k_end = min(g.K, k0 + g.k_per);
    const int steps = (k_end - k0 + kStep - 1) / kStep, whole = (k_end - k0) / kStep;
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);

    using TileA = Tile4<BM, W, G>;
    using TileB = Tile4<BN, W, G>;
    constexpr int kLoads = TileA::kLoads + TileB::kLoads + 1;
    TileA ta;
    TileB tb;
    S ts;
    ta.setup((uint32_t)g.lda * 2, g.M - m0, wave, lane);
    tb.setup((uint32_t)g.ldb * 2, g.N - n0, wave, lane);
    ts.setup(scales, (uint32_t)m0, (uint32_t)n0, k0 / 32, wave, lane);
    const char *pa = (const char *)g.a + ((int64_t)m0 * g.lda + k0) * 2;
    const char *pb = (const char *)g.b + ((int64_t)n0 * g.ldb + k0) * 2;

    f32x16 acc[TN][TM];
    each<TN * TM>([&](auto x) __attribute__((always_inline)) { acc[x % TN][x / TN] = f32x16{}; });
    u32x4 fa[2][TM], fb[2][TN];
    uint32_t sa[TM], sb[TN], sa_last[TM], sb_last[TN];         // of this step, and of the one whose last pair is still to come
#pragma unroll
    for (int j = 0; j < TM; ++j) fa[1][j] = u32x4{0, 0, 0, 0}, sa[j] = 0;
#pragma unroll
    for (int i = 0; i < TN; ++i) fb[1][i] = u32x4{0, 0, 0, 0}, sb[i] = 0;

    // loads of one step, in order of steps; all of it is there (WHOLE) or zeros stand for what is not
    auto issue = [&](auto all, int s, char *to) {
        constexpr bool WHOLE = decltype(all)::value;
        const int left = WHOLE ? G : (k_end - k0) / 32 - s * G;
        ta.template load<WHOLE>(pa, to, left, wave);
        tb.template load<WHOLE>(pb, to + kA, left, wave);
        ts.load(to + kA + kB, left);
        pa += 64 * G;
        pb += 64 * G;
    };
    auto read = [&](const char *from, int q) {
#pragma unroll
        for (int i = 0; i < TN; ++i) fb[q & 1][i] = TileB::read(from + kA, wn + 32 * i, q, lane);
#pragma unroll
        for (int j = 0; j < TM; ++j) fa[q & 1][j] = TileA::read(from, wm + 32 * j, q, lane);
    };
    auto read_scales = [&](const char *from) {
        const char *words = from + kA + kB;
#pragma unroll
        for (int j = 0; j < TM; ++j) sa_last[j] = sa[j], sa[j] = S::template read<BM>(words, wm + 32 * j, lane);
#pragma unroll
        for (int i = 0; i < TN; ++i) sb_last[i] = sb[i], sb[i] = S::template read<BN>(words + S::kX * 1024, wn + 32 * i, lane);
    };
    // the matrix instructions first .. last - 1 of pair q, by the scales of this step or of the one before
    auto multiply = [&](auto q, auto before, auto first, auto last) __attribute__((always_inline)) {
        each<last - first>([&](auto y) __attribute__((always_inline)) {
            constexpr int x = first + y, i = x % TN, j = x / TN, Q = decltype(q)::value, set = Q & 1;
            const int a = decltype(before)::value ? (int)sa_last[j] : (int)sa[j], b = decltype(before)::value ? (int)sb_last[i] : (int)sb[i];
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand4(fb[set][i]), operand4(fa[set][j]), acc[i][j], 4, 4,
                                                                        Q, b, Q, a);
        });
    };
    constexpr int kAll = TM * TN, kHalf = kAll / 2;
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, kPairs - 1> cLastPair{};
    constexpr std::integral_constant<int, kHalf> cHalf{};
    constexpr std::integral_constant<int, kAll> cAll{};
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    // the order of a run of matrix instructions and of what goes behind them: the LDS reads, two after each at least, and
    // the next loads, spread over the step's first one and a half pairs
    auto order = [&](auto count, auto with_loads, auto with_scales) {
        constexpr int kReads = TM + TN + (decltype(with_scales)::value ? G * (TM + TN) : 0);
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
        read_scales(from);
        read(from, 0);
        multiply(cLastPair, yes, cHalf, cAll);
        if (decltype(all)::value || s - 1 + BUF < steps) issue(all, s - 1 + BUF, to);
        order(std::integral_constant<int, kAll - kHalf>{}, all, yes);
        each<kPairs - 1>([&](auto q) __attribute__((always_inline)) {
            read(from, q + 1);
            multiply(q, no, c0, cAll);
            if constexpr (decltype(all)::value && decltype(q)::value == 0) order(cAll, yes, no);
            else order(cAll, no, no);
        });
        multiply(cLastPair, no, c0, cHalf);
    };
#pragma unroll
    for (int s = 0; s < BUF - 1; ++s)
        if (s < whole) issue(yes, s, lds[s]);
        else if (s < steps) issue(no, s, lds[s]);
    if (steps >= BUF - 1) turn<(BUF - 2) * kLoads>();
    else turn<0>();
    // step s's loads are this wave's oldest: they have landed when no more than those of the steps after it are on their
    // way; behind the barrier everybody's have, and nobody reads the buffer of step s - 1 any more
    int fill = BUF - 1, from = 0, s = 0;
    for (; s - 1 + BUF < whole; ++s) {
        step(yes, lds[fill], lds[from], s);
        turn<(BUF - 2) * kLoads>();
        fill = from;
        from = from + 1 == BUF ? 0 : from + 1;
    }
    for (; s < steps; ++s) {
        step(no, lds[fill], lds[from], s);
        turn<0>();
        fill = from;
        from = from + 1 == BUF ? 0 : from + 1;
    }
    multiply(cLastPair, no, cHalf, cAll);

    // (f32: half as many rows at a time, or the residual's registers would not fit beside the sums)
    constexpr int R = sizeof(T) == 2 ? 32 : 16, kParts = 32 / R;
    float *piece = (float *)lds + wave * 32 * kOutPitch;
    store_wave<T, R, TM * TN / 2 * kParts, false>(piece, g, e, lane,
        [&](int x) __attribute__((always_inline)) {  // (one copy of the epilogue's code, whichever the accumulators)
            each<TM * TN / 2>([&](auto y) __attribute__((always_inline)) {
                if (x / kParts == y && (kParts == 1 || ((lane & 31) / R) == x % kParts))
                    each<2>([&](auto i) __attribute__((always_inline)) {
                        f32x16 a = acc[y / TM * 2 + i][y % TM];
                        asm volatile("" : "+v"(a));   // (or the compiler joins the branches by the accumulators' addresses)
                        each<4>([&](auto z) __attribute__((always_inline)) {
                            constexpr int q = 4 * z;
                            *(f32x4 *)(piece + (lane & (R - 1)) * kOutPitch + 32 * i + 2 * q + (lane >> 5) * 4) =
                                f32x4{a[q], a[q + 1], a[q + 2], a[q + 3]};
                        });
                    });
            });
        },
        [&](int x) __attribute__((always_inline)) {
            const int y = x / kParts;
            return int2{m0 + wm + y % TM * 32 + x % kParts * R, n0 + wn + y / TM * 64};
        });
}

}  // namespace tvl
