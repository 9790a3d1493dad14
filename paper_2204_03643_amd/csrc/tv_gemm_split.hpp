// Matrix products on operands of any alignment, and on f32 operands: tiles pass through registers on their way to LDS,
// and f32 values are split there into three bf16 parts,
//     x = h + m + l,   h = bf16(x), m = bf16(x - h), l = bf16(x - h - m):
// three times eight bits hold the 24 of an f32, and a product is the sum of the six partial products whose orders add
// up to two at most (h h, h m, m h, h l, m m, l h); the three that are left out are below 2^-24 of it together.
// Six bf16 matrix instructions do the work of eight f32 ones in 0.38 of their time.  An operand of restored 8-bit codes is
// exact in bf16 and has one part: three products.
//
// That holds for magnitudes of 2^-110 and more (and zero).  Below, the last bits of m and l are below bf16's least number,
// 2^-133, and a value is taken to half of that, 2^-134: a product is then off by up to 2^-134 times the other value.  (Telling
// such values while they are split takes one and a half instructions a value beside 5.5, and would send every tile that holds
// one among larger values, where it does not count, to the slow f32 instructions.)
//
// Splitting is vector work that the matrix units do not hide in full: 8192 x 2048 -> 8192 takes 1.19 ms (231 TFLOP/s of f32
// products, 1.4 PFLOP/s of bf16 ones); 128 x 128 outputs take 1.8 us a step of 64 where up to half of the compute units have a
// tile, 2.6 where all have (4096 x 1024 -> 1024: 49 us, 175 TFLOP/s, the matrix units busy for 0.57 of the cycles).  bf16 operands off 16-byte boundaries pay for their way through
// registers: 505 us for 8192 x 2047 -> 8191.
//
// A part of an infinity, or of a value beyond bf16's largest, times zero is a NaN that the f32 product need not be, and
// parts that were rounded up may multiply to an infinity where the f32 product is finite: a wave that finds a sum that is not
// finite among its own takes it from f32 matrix instructions.
#pragma once
#include "tv_gemm16.hpp"

namespace tvl {

// The two values next to one another, the first in the lower half.
__device__ __forceinline__ uint32_t narrow2(float x, float y)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
}

template <class T> struct Parts { static constexpr int kCount = sizeof(T) == 4 ? 3 : 1; };

// ROWS output indices by 16 KQ contraction indices of an operand, on its way through THREADS threads: eight consecutive
// elements a unit, 16 bytes of each part in LDS.
//
// k contiguous: 32 KQ bytes a row, its 16-byte piece c in slot c ^ (r KQ / 8) % (2 KQ): sixteen rows read at one c touch
// all banks once.  transposed: as Tile16 has it.
template <class T, int ROWS, int THREADS, int KQ, bool TRANSPOSED> struct Staged {
    static constexpr int kParts = Parts<T>::kCount, kUnits = ROWS * KQ * 2 / THREADS, kBytes = ROWS * KQ * 32;   // of a part
    static constexpr int kRaw = sizeof(T) == 4 ? 2 : 1, E = Elems<T>::kPer16;
    static_assert(kUnits >= 1 && kUnits * THREADS == ROWS * KQ * 2, "");
    struct Raw { u32x4 v[kUnits][kRaw]; };
    const T *from[kUnits];       // of the step whose turn it is

    __device__ __forceinline__ static int swizzle(int kk) { return ROWS >= 128 ? (kk & 3) << 2 : (kk & 2) << 1; }

    // (k contiguous: a row beyond the last one stands for it, its outputs are not kept)
    __device__ __forceinline__ void setup(const T *p, int64_t ld, int rows, int row0, int k0, int t)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = t + u * THREADS;
            if constexpr (!TRANSPOSED) from[u] = p + (int64_t)min(row0 + at / (2 * KQ), rows - 1) * ld + k0 + at % (2 * KQ) * 8;
            else from[u] = p + (int64_t)(k0 + at / (ROWS / 8)) * ld + row0 + at % (ROWS / 8) * 8;
        }
    }
    // WHOLE: everything is there.  Otherwise zeros stand for what is beyond the contraction's end (k: the step's first index)
    // and, transposed, beyond the last row.
    template <bool WHOLE>
    __device__ __forceinline__ void load(Raw &raw, int64_t ld, int rows, int k_end, int row0, int k, int t)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = t + u * THREADS;
            int have = 8;
            if constexpr (!WHOLE) {
                if constexpr (!TRANSPOSED) have = k_end - (k + at % (2 * KQ) * 8);
                else have = k + at / (ROWS / 8) < k_end ? rows - (row0 + at % (ROWS / 8) * 8) : 0;
            }
#pragma unroll
            for (int i = 0; i < kRaw; ++i) raw.v[u][i] = load16(from[u] + i * E, WHOLE ? E : have - i * E);
            from[u] += TRANSPOSED ? 16 * KQ * ld : 16 * KQ;
        }
    }
    __device__ __forceinline__ static void put(const Raw &raw, char *lds, int t)
    {
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            const int at = t + u * THREADS;
            char *to;
            if constexpr (!TRANSPOSED) {
                const int r = at / (2 * KQ), c = at % (2 * KQ);
                to = lds + r * (32 * KQ) + ((c ^ (r * KQ / 8 % (2 * KQ))) << 4);
            } else {
                const int kk = at / (ROWS / 8), c = at % (ROWS / 8);
                to = lds + kk * (ROWS * 2) + ((c ^ swizzle(kk)) << 4);
            }
            if constexpr (sizeof(T) == 2) *(u32x4 *)to = raw.v[u][0];
            else {
                u32x4 part[3];
#pragma unroll
                for (int i = 0; i < 4; ++i) {          // (one instruction rounds two values)
                    float x = __uint_as_float(raw.v[u][i >> 1][i * 2 & 2]), y = __uint_as_float(raw.v[u][i >> 1][(i * 2 & 2) + 1]);
#pragma unroll
                    for (int j = 0; j < 3; ++j) {
                        const uint32_t two = narrow2(x, y);
                        part[j][i] = two;
                        x -= __uint_as_float(two << 16);
                        y -= __uint_as_float(two & 0xffff0000u);
                    }
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) *(u32x4 *)(to + j * kBytes) = part[j];
            }
        }
    }
    // as Tile16::read, of one part
    __device__ __forceinline__ static bf16x8 read(const char *lds, int row, int q, int lane)
    {
        if constexpr (!TRANSPOSED) {
            const int r = row + (lane & 31), c = q * 2 + (lane >> 5);
            return *(const bf16x8 *)(lds + r * (32 * KQ) + ((c ^ (r * KQ / 8 % (2 * KQ))) << 4));
        } else {
            const int kk = q * 16 + (lane >> 5) * 8 + ((lane >> 2) & 3);
            const int col = row + (lane & 16) + (lane & 3) * 4;
            const char *p = lds + kk * (ROWS * 2) + (((col >> 3) ^ swizzle(kk)) << 4) + (col & 4) * 2;
            typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * ROWS * 2));
            typedef int16_t s16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// A 32 x 32 tile of outputs from (m0, n0) on with f32 matrix instructions, two contraction indices at a time, straight
// from memory: what is left for tiles with sums that are not finite.
template <class TA, class TB, bool AT, bool BT>
__device__ __attribute__((noinline)) f32x16 tile_in_f32(const TA *a, const TB *b, int64_t lda, int64_t ldb, int M, int N, int k0, int k_end, int m0, int n0, int lane)
{
    const int64_t m = min(m0 + (lane & 31), M - 1), n = min(n0 + (lane & 31), N - 1);
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
    for (int k = k0; k < k_end; k += 2) {
        const int64_t kk = min(k + (lane >> 5), k_end - 1);
        const bool there = k + (lane >> 5) < k_end;
        const float x = widen(a[AT ? kk * lda + m : m * lda + kk]), y = widen(b[BT ? kk * ldb + n : n * ldb + kk]);
        acc = __builtin_amdgcn_mfma_f32_32x32x2f32(there ? y : 0.0f, there ? x : 0.0f, acc, 0, 0, 0);
    }
    return acc;
}

// T: A's type and the outputs'; TB: B's.
// G: groups of waves that share out a step's contraction, each with sums of its own for all outputs; they are joined in LDS at
// the end.  (A small tile has few waves; two groups keep the matrix units busy where one waits: 1024 x 1024
// over 1024 in tiles of 64 x 128 took 29 us with one group of four waves, 26 with two.)
template <class T, class TB, int BM, int BN, int WM, int WN, int KQ, int AHEAD, int G, bool AT, bool BT>
__global__ __launch_bounds__(WM * WN * G * 64) __attribute__((amdgpu_waves_per_eu(2))) void gemm_split_kernel(Product g, Epilogue e)
{
    constexpr int W = WM * WN, THREADS = W * G * 64, TM = BM / WM / 32, TN = BN / WN / 32, P = Parts<T>::kCount, PB = Parts<TB>::kCount;
    constexpr int kOrders = P > PB ? P : PB;
    using TileA = Staged<T, BM, THREADS, KQ, AT>;
    using TileB = Staged<TB, BN, THREADS, KQ, BT>;
    constexpr int kA = P * TileA::kBytes, kB = PB * TileB::kBytes, kOut = W * 32 * kOutPitch * 4;
    constexpr int kJoin = G > 1 ? (G - 1) * BM * BN * 4 : 0;
    static_assert(TN % 2 == 0, "a wave's outputs leave 64 columns at a time");
    static_assert(KQ % G == 0 && kJoin <= 2 * (kA + kB), "");
    __shared__ __attribute__((aligned(1024))) char lds[2 * (kA + kB) > kOut ? 2 * (kA + kB) : kOut];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    uint32_t tm, tn;
    tile_of(blockIdx.x, g.tiles_m, g.tiles_n, tm, tn);
    // (a transposed operand's last tile starts early enough to be whole: its first outputs are the tile before's too, to
    // the bit, and a tile that reads past the last row would load element by element)
    const int m0 = AT ? min((int)tm * BM, max(0, g.M - BM)) : (int)tm * BM;
    const int n0 = BT ? min((int)tn * BN, max(0, g.N - BN)) : (int)tn * BN;
    const int k0 = (int)blockIdx.y * g.k_per, k_end = min(g.K, k0 + g.k_per);
    const int steps = (k_end - k0 + 16 * KQ - 1) / (16 * KQ);
    const int group = wave / W, wm = wave % WM * (BM / WM), wn = wave % W / WM * (BN / WN);

    f32x16 acc[TN][TM];
    each<TN * TM>([&](auto x) __attribute__((always_inline)) { acc[x % TN][x / TN] = f32x16{}; });

    // AHEAD steps' values are in registers or on their way besides the two in LDS; past the contraction's end there are zeros
    TileA ta;
    TileB tb;
    ta.setup((const T *)g.a, g.lda, g.M, m0, k0, t);
    tb.setup((const TB *)g.b, g.ldb, g.N, n0, k0, t);
    struct Both { typename TileA::Raw a; typename TileB::Raw b; } raw[AHEAD];
    auto load = [&](auto all, Both &r, int s) {
        constexpr bool WHOLE = decltype(all)::value;
        ta.template load<WHOLE>(r.a, g.lda, g.M, k_end, m0, k0 + s * 16 * KQ, t);
        tb.template load<WHOLE>(r.b, g.ldb, g.N, k_end, n0, k0 + s * 16 * KQ, t);
    };
    auto put = [&](const Both &r, char *to) {
        TileA::put(r.a, to, t);
        TileB::put(r.b, to + kA, t);
    };
    auto step = [&](auto which, Both &r, const char *from, char *to, int s) {
#pragma unroll
        for (int i = 0; i < KQ / G; ++i) {
            const int q = group * (KQ / G) + i;
            bf16x8 fa[P][TM], fb[PB][TN];
#pragma unroll
            for (int o = 0; o < PB; ++o)
#pragma unroll
                for (int i = 0; i < TN; ++i) fb[o][i] = TileB::read(from + kA + o * TileB::kBytes, wn + 32 * i, q, lane);
#pragma unroll
            for (int o = 0; o < P; ++o)
#pragma unroll
                for (int j = 0; j < TM; ++j) fa[o][j] = TileA::read(from + o * TileA::kBytes, wm + 32 * j, q, lane);
            // by their order's size, the smallest first
            each<kOrders>([&](auto z) __attribute__((always_inline)) {
                constexpr int order = kOrders - 1 - z, first = order < PB ? 0 : order - PB + 1, last = order < P ? order : P - 1;
                each<last - first + 1>([&](auto y) __attribute__((always_inline)) {
                    constexpr int oa = first + y, ob = order - oa;
                    each<TM * TN>([&](auto x) __attribute__((always_inline)) {
                        constexpr int i = x % TN, j = x / TN;
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[ob][i], fa[oa][j], acc[i][j], 0, 0, 0);
                    });
                });
            });
        }
        put(r, to);
        load(which, r, s + 1 + AHEAD);
        if constexpr (AHEAD > 1) {
            constexpr int kReads = KQ / G * (P * TM * (AT ? 2 : 1) + PB * TN * (BT ? 2 : 1));
            constexpr int kMfma = (P * PB > 3 ? 6 : P * PB) * (KQ / G) * TM * TN;
            constexpr int kSplit = TileA::kUnits * (P > 1 ? 60 : 8) + TileB::kUnits * (PB > 1 ? 60 : 8), kEach = (kSplit + kMfma - 1) / kMfma;
            __builtin_amdgcn_sched_group_barrier(0x100, kReads / (KQ / G), 0);
#pragma unroll
            for (int x = 0; x < kMfma; ++x) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, kEach, 0);
                if (x * 2 < kReads - kReads / (KQ / G)) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
        }
        __syncthreads();
    };
    char *even = lds, *odd = lds + kA + kB;
    const std::false_type some;
    const std::true_type all;
    const bool inside = (!AT || m0 + BM <= g.M) && (!BT || n0 + BN <= g.N);
    const int whole = inside ? (k_end - k0) / (16 * KQ) : 0;
    auto first = [&](auto all_or_some) {
        load(all_or_some, raw[0], 0);
        put(raw[0], even);
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) load(all_or_some, raw[(s + 1) % AHEAD], s + 1);
    };
    if (AHEAD < whole) first(all);
    else first(some);
    __syncthreads();
    int s = 0;
    for (; s + 2 + AHEAD < whole; s += 2) {
        step(all, raw[1 % AHEAD], even, odd, s);
        step(all, raw[0], odd, even, s + 1);
    }
    for (; s < steps; s += 2) {
        step(some, raw[1 % AHEAD], even, odd, s);
        step(some, raw[0], odd, even, s + 1);
    }
    if constexpr (G > 1) {
        // sum by sum, so that a wave's lanes write side by side
        float *mine = (float *)lds + (wave % W) * (TM * TN * 16 * 64) + lane;
        each<G - 1>([&](auto y) __attribute__((always_inline)) {
            constexpr int from = y + 1;
            float *there = mine + y * (BM * BN);
            if (group == from)
                each<TM * TN>([&](auto x) __attribute__((always_inline)) {
                    each<16>([&](auto q) __attribute__((always_inline)) { there[(x * 16 + q) * 64] = acc[x % TN][x / TN][decltype(q)::value]; });
                });
        });
        __syncthreads();
        if (group == 0)
            each<G - 1>([&](auto y) __attribute__((always_inline)) {
                const float *there = mine + y * (BM * BN);
                each<TM * TN>([&](auto x) __attribute__((always_inline)) {
                    each<16>([&](auto q) __attribute__((always_inline)) { acc[x % TN][x / TN][decltype(q)::value] += there[(x * 16 + q) * 64]; });
                });
            });
        __syncthreads();
        if (group) return;                            // (no barrier comes after this)
    }
    if constexpr (P * PB > 1) {
        uint32_t most = 0;                            // of all sums, the bits of what is not finite being above the others'
        each<TM * TN>([&](auto x) __attribute__((always_inline)) {
            each<16>([&](auto q) __attribute__((always_inline)) {
                most = max(most, __float_as_uint(acc[x % TN][x / TN][decltype(q)::value]) & 0x7fffffffu);
            });
        });
        if (__any(most >= 0x7f800000u))
            each<TM * TN>([&](auto x) __attribute__((always_inline)) {
                constexpr int i = x % TN, j = x / TN;
                const f32x16 again = tile_in_f32<T, TB, AT, BT>((const T *)g.a, (const TB *)g.b, g.lda, g.ldb, g.M, g.N, k0, k_end,
                                                                m0 + wm + 32 * j, n0 + wn + 32 * i, lane);
                each<16>([&](auto y) __attribute__((always_inline)) {
                    constexpr int q = y;
                    const bool finite = (__float_as_uint(acc[i][j][q]) & 0x7fffffffu) < 0x7f800000u;
                    acc[i][j][q] = finite ? acc[i][j][q] : again[q];
                });
            });
    }
    float *piece = (float *)lds + wave * 32 * kOutPitch;
    store_wave<T, 32, TM * TN / 2, AT || BT>(piece, g, e, lane,
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
