// Products of values in 4 bits on tiles: D[m, n] = sum_k X(m, k) W(n, k), both in blocks of 32 with a scale each.
//
// A block's 16 bytes of codes are what a lane hands to a scaled matrix instruction (32 x 32 x 64), so that the tiles are those
// of 16-bit products byte for byte: 128 bytes a row are a step of 256 values here.  The scales come beside them, a word of
// four for each group of 128, and a lane picks its four of a step with one permutation.
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

// Where a tile's scale words come from.  A wave loads 1024 bytes a step: 256 rows' words of a group, or those of both groups of
// the step one after the other.  What is needed are kParts such pieces; further waves load one of them again, so that
// all waves have as many loads on their way.
template <int BM, int BN> struct Scales4 {
    static constexpr int kX = BM == 256 ? 2 : 1, kW = BN == 256 ? 2 : 1, kParts = kX + kW;
    const char *from;
    int64_t step;            // bytes to the next step
    int32_t back;            // bytes from this lane's word of a step's second group to that of its first; 0 in the first

    __device__ __forceinline__ void setup(const Scales &s, uint32_t m0, uint32_t n0, int first, int wave, int lane)
    {
        const int part = wave % kParts;
        const bool of_x = part < kX;
        const int rows = of_x ? BM : BN, piece = of_x ? part : part - kX;
        const uint32_t pitch = of_x ? s.x_rows : s.w_rows;
        const int at = lane * 4, group = rows == 256 ? piece : at / rows & 1;
        const uint32_t row = min((of_x ? m0 : n0) + (uint32_t)(at % rows), pitch - 4);
        from = (const char *)((of_x ? s.x : s.w) + ((int64_t)first + group) * pitch + row);
        step = (int64_t)pitch * 8;
        back = group ? (int32_t)(pitch * 4) : 0;
    }
    // groups: how many are left from the step on
    __device__ __forceinline__ void load(char *lds, int groups, int wave)
    {
        const char *p = groups >= 2 ? from : from - (uint32_t)back;
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p,
                                         (__attribute__((address_space(3))) void *)(lds + wave * 1024), 16, 0, 0);
        from += step;
    }
    // The scales of 32 rows from `row` on: lane l has those of row l % 32, byte q that of block 2 q + l / 32 of the step.
    template <int ROWS> __device__ __forceinline__ static uint32_t read(const char *words, int row, int lane)
    {
        const uint32_t *w = (const uint32_t *)words + row + (lane & 31);
        return __builtin_amdgcn_perm(w[ROWS], w[0], lane < 32 ? 0x06040200u : 0x07050301u);
    }
};

// BM x BN outputs a workgroup of WM x WN waves, BUF buffers of a step; the order of things is gemm16_kernel's.  g counts
// codes by twos of bytes: lda, ldb and K are 32 a group.
template <class T, int BM, int BN, int WM, int WN, int BUF>
__global__ __launch_bounds__(WM * WN * 64) void gemm4_kernel(Product g, Scales scales, Epilogue e)
{
    constexpr int W = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kA = BM * 128, kB = BN * 128, kS = W * 1024, kOut = W * 32 * kOutPitch * 4;
    using S = Scales4<BM, BN>;
    static_assert(TN % 2 == 0, "a wave's outputs leave 64 columns at a time");
    static_assert(W >= S::kParts, "the waves load all scales");
    static_assert(kOut <= BUF * (kA + kB + kS), "the outputs' pieces fit");
    __shared__ __attribute__((aligned(1024))) char lds[BUF][kA + kB + kS];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    const int m0 = (int)tm * BM, n0 = (int)tn * BN;
    const int k0 = (int)blockIdx.y * g.k_per, k_end = min(g.K, k0 + g.k_per);
    const int steps = (k_end - k0 + 63) / 64, whole = (k_end - k0) / 64;
    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);

    using TileA = Tile16<BM, W, false>;
    using TileB = Tile16<BN, W, false>;
    constexpr int kLoads = TileA::kLoads + TileB::kLoads + 1;
    TileA ta;
    TileB tb;
    S ts;
    ta.setup((uint32_t)g.lda, g.M - m0, wave, lane);
    tb.setup((uint32_t)g.ldb, g.N - n0, wave, lane);
    ts.setup(scales, (uint32_t)m0, (uint32_t)n0, k0 / 32, wave, lane);
    const char *pa = (const char *)g.a + ((int64_t)m0 * g.lda + k0) * 2;
    const char *pb = (const char *)g.b + ((int64_t)n0 * g.ldb + k0) * 2;

    f32x16 acc[TN][TM];
    each<TN * TM>([&](auto x) __attribute__((always_inline)) { acc[x % TN][x / TN] = f32x16{}; });
    u32x4 fa[2][TM], fb[2][TN];
    uint32_t sa[TM], sb[TN], sa_last[TM], sb_last[TN];         // of this step, and of the one whose last block is still to come
#pragma unroll
    for (int j = 0; j < TM; ++j) fa[1][j] = u32x4{0, 0, 0, 0}, sa[j] = 0;
#pragma unroll
    for (int i = 0; i < TN; ++i) fb[1][i] = u32x4{0, 0, 0, 0}, sb[i] = 0;

    auto issue = [&](auto all, int s, char *to) {
        constexpr bool WHOLE = decltype(all)::value;
        const int left = k_end - k0 - s * 64;
        ta.template load<WHOLE>(pa, to, left, wave);
        tb.template load<WHOLE>(pb, to + kA, left, wave);
        ts.load(to + kA + kB, WHOLE ? 2 : left / 32, wave);
        pa += 128;
        pb += 128;
    };
    auto read = [&](const char *from, int q, int set) {
#pragma unroll
        for (int i = 0; i < TN; ++i) fb[set][i] = __builtin_bit_cast(u32x4, TileB::read(from + kA, wn + 32 * i, q, lane));
#pragma unroll
        for (int j = 0; j < TM; ++j) fa[set][j] = __builtin_bit_cast(u32x4, TileA::read(from, wm + 32 * j, q, lane));
    };
    auto read_scales = [&](const char *from) {
        const char *words = from + kA + kB;
#pragma unroll
        for (int j = 0; j < TM; ++j) sa_last[j] = sa[j], sa[j] = S::template read<BM>(words, wm + 32 * j, lane);
#pragma unroll
        for (int i = 0; i < TN; ++i) sb_last[i] = sb[i], sb[i] = S::template read<BN>(words + S::kX * 1024, wn + 32 * i, lane);
    };
    // the matrix instructions first .. last - 1 of block pair q, by the scales of this step or (LAST) of the one before
    auto multiply = [&](auto q, auto last_step, auto first, auto last) __attribute__((always_inline)) {
        each<last - first>([&](auto y) __attribute__((always_inline)) {
            constexpr int x = first + y, i = x % TN, j = x / TN, Q = decltype(q)::value, set = Q & 1;
            const int a = decltype(last_step)::value ? (int)sa_last[j] : (int)sa[j], b = decltype(last_step)::value ? (int)sb_last[i] : (int)sb[i];
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand4(fb[set][i]), operand4(fa[set][j]), acc[i][j], 4, 4,
                                                                        Q, b, Q, a);
        });
    };
    constexpr int kAll = TM * TN, kHalf = kAll / 2;
    constexpr std::integral_constant<int, 0> c0{};
    constexpr std::integral_constant<int, 1> c1{};
    constexpr std::integral_constant<int, 2> c2{};
    constexpr std::integral_constant<int, 3> c3{};
    constexpr std::integral_constant<int, kHalf> cHalf{};
    constexpr std::integral_constant<int, kAll> cAll{};
    auto order = [&](auto count, auto with_loads, auto with_scales) {
        constexpr int kReads = TM + TN + (decltype(with_scales)::value ? 2 * (TM + TN) : 0);
        constexpr int n = decltype(count)::value, kEach = (kReads + n - 1) / n > 2 ? (kReads + n - 1) / n : 2;
        constexpr int kLoadsEach = (kLoads + kAll + kHalf - 1) / (kAll + kHalf);
#pragma unroll
        for (int x = 0; x < n; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (x * kEach < kReads) __builtin_amdgcn_sched_group_barrier(0x100, kEach, 0);
            if constexpr (decltype(with_loads)::value) __builtin_amdgcn_sched_group_barrier(0x010, kLoadsEach, 0);
        }
    };
    auto step = [&](auto all, char *__restrict to, const char *__restrict from, int s) {
        read_scales(from);
        read(from, 0, 0);
        multiply(c3, std::true_type{}, cHalf, cAll);
        if (decltype(all)::value || s - 1 + BUF < steps) issue(all, s - 1 + BUF, to);
        order(std::integral_constant<int, kAll - kHalf>{}, all, std::true_type{});
        read(from, 1, 1);
        multiply(c0, std::false_type{}, c0, cAll);
        order(cAll, all, std::false_type{});
        read(from, 2, 0);
        multiply(c1, std::false_type{}, c0, cAll);
        order(cAll, std::false_type{}, std::false_type{});
        read(from, 3, 1);
        multiply(c2, std::false_type{}, c0, cAll);
        order(cAll, std::false_type{}, std::false_type{});
        multiply(c3, std::false_type{}, c0, cHalf);
    };
#pragma unroll
    for (int s = 0; s < BUF - 1; ++s)
        if (s < whole) issue(std::true_type{}, s, lds[s]);
        else if (s < steps) issue(std::false_type{}, s, lds[s]);
    if (steps >= BUF - 1) turn<(BUF - 2) * kLoads>();
    else turn<0>();
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
    multiply(c3, std::false_type{}, cHalf, cAll);

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
