// The border between two residual blocks: y = x + d scale act(gate) norm(f), h = next_norm(y), and its gradients.
//
// Reads and writes are all there is to it: a row is read once, its statistics are taken of what the lanes hold, and what
// follows from them is written.  Lanes side by side in a row hold eight neighbouring channels each.  In bf16, microseconds
// (GB/s read + written): norm of 8192 x 2048 12.7 (5300), its gradients 19.3 (5200) and the join of the weight's 4.8; border of 16384 x 2048
// with norms, a gate a sequence, scale and dropout 52 (5100), its gradients 92 (4400) and the join 7.1.
#pragma once
#include "tv_block_plan.hpp"
#include "tv_drop.hpp"

namespace tvl {

enum Norm : int { kNormNone = 0, kNormRms = 1, kNormLayer = 2 };
enum Gate : int { kGatePlain = 0, kGateSigmoid = 1, kGateSilu = 2 };

struct Block {
    const void *x, *f, *w, *b, *gate, *scale, *nw, *nb;
    int64_t m, ldx, ldf, ldg;
    int32_t n, gate_div, norm, next, act;
    bool    again;           // backward: y is made again of x and f (bf16)
    float   eps, inv_n;
    Drop    drop;
};

// Sums over LANES lanes of a wave, in all of them: neighbours, pairs, quads and eights by moves within sixteen lanes, then the
// sixteens and halves of the wave by exchanging them.
template <int CTRL> __device__ __forceinline__ float lanes_moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LANES> __device__ __forceinline__ float wave_sum(float v)
{
    v += lanes_moved<0xB1>(v);                       // [1, 0, 3, 2]
    v += lanes_moved<0x4E>(v);                       // [2, 3, 0, 1]
    v += lanes_moved<0x141>(v);                      // mirrored within 8
    if constexpr (LANES > 8) v += lanes_moved<0x140>(v);      // within 16
    if constexpr (LANES > 16) {
        const auto o = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(o[0]) + __uint_as_float(o[1]);
    }
    if constexpr (LANES > 32) {
        const auto o = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(o[0]) + __uint_as_float(o[1]);
    }
    return v;
}

// A value that is the same in all lanes of a wave, out of the vector registers.
__device__ __forceinline__ float of_wave(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }

// Sums over the LANES lanes of a row.  More than a wave: through LDS, in two places in turn, so that one barrier a sum is
// enough (between the read of a place and its next write lies the barrier of the sum in between).
template <int LANES> struct RowSum {
    static constexpr int kWaves = LANES > 64 ? LANES / 64 : 1;
    float2 (*place)[kWaves];
    int turn = 0;
    __device__ __forceinline__ explicit RowSum(float2 (*lds)[kWaves]) : place(lds) {}
    __device__ __forceinline__ float2 operator()(float a, float b)
    {
        constexpr int kLanes = LANES < 64 ? LANES : 64;
        a = wave_sum<kLanes>(a);
        b = wave_sum<kLanes>(b);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) place[turn][threadIdx.x >> 6] = float2{a, b};
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                a += place[turn][i].x;
                b += place[turn][i].y;
            }
            turn ^= 1;
        }
        return {a, b};
    }
    __device__ __forceinline__ float operator()(float a)
    {
        a = wave_sum<LANES < 64 ? LANES : 64>(a);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) place[turn][threadIdx.x >> 6].x = a;
            __syncthreads();
            a = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) a += place[turn][i].x;
            turn ^= 1;
        }
        return a;
    }
};

// act(z).
template <bool FAST> __device__ __forceinline__ float gate_of(float z, int act)
{
    if (act == kGateSigmoid) return logistic<FAST>(z);
    if (act == kGateSilu) return z * logistic<FAST>(z);
    return z;
}
// act(z) in place of eight z, which one is asked once for all of them.
template <bool FAST> __device__ __forceinline__ void gate8(float (&z)[8], int act)
{
    if (act == kGateSigmoid)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = logistic<FAST>(z[i]);
    else if (act == kGateSilu)
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= logistic<FAST>(z[i]);
}
// The same, and the eight values of v times act's slope; four at a time, which takes fewer registers.
template <bool FAST> __device__ __forceinline__ void gate8(float (&z)[8], float (&v)[8], int act)
{
    if (act == kGateSigmoid)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = logistic<FAST>(z[i]);
            v[i] *= s * (1.0f - s);
            z[i] = s;
            if (i == 3) __builtin_amdgcn_sched_barrier(0);
        }
    else if (act == kGateSilu)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = logistic<FAST>(z[i]);
            v[i] *= s * (1.0f + z[i] * (1.0f - s));
            z[i] *= s;
            if (i == 3) __builtin_amdgcn_sched_barrier(0);
        }
}

template <class T> __device__ __forceinline__ void load_or(float (&v)[8], const void *p, int col, int have, float otherwise)
{
    if (p) get8(v, (const T *)p + col, have);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = otherwise;
}

// Eight neighbouring values as they lie in memory.
template <class T> struct Raw8 {
    u32x4 v[sizeof(T) / 2];
    __device__ __forceinline__ float operator[](int i) const
    {
        if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? v[0][i >> 1] & 0xffff0000u : v[0][i >> 1] << 16);
        else return __uint_as_float(v[i >> 2][i & 3]);
    }
};
// The channels of a lane: `have` from `col` on.  Without a TAIL that is eight.  A row's last lane may have fewer, and loads
// the row's last eight, `back` before its own, to move them down: the same accesses as the other lanes', and none beyond the row
// (16384 x 2047 bf16: 134 us with its last values one by one, 73 so; 50 for 2040 channels, without a tail).
struct Cols {
    int col, have, back;
};
template <bool TAIL> __device__ __forceinline__ Cols cols_of(int lane, int n)
{
    const bool live = lane * 8 < n;
    Cols c{TAIL || live ? lane * 8 : 0, 8, 0};
    if constexpr (TAIL) {
        c.have = max(0, min(8, n - c.col));
        c.back = c.have > 0 && n >= 8 ? 8 - c.have : 0;
    }
    return c;
}

// Asks for eight values of a row that starts at p; settle8 makes of them, once they are there, the lane's own and zeros for those
// that do not exist.  (Apart, or whoever asks ahead of time would wait.)
template <bool TAIL, class T> __device__ __forceinline__ Raw8<T> raw8(const T *p, Cols c)
{
    Raw8<T> r;
    if (!TAIL || c.have == 8 || c.back) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = get16(p + c.col - c.back + i * (16 / (int)sizeof(T)));
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = u32x4{0, 0, 0, 0};
        if (c.have)                                  // a row of fewer than eight
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const T v = p[min(i, c.have - 1)];
                if constexpr (sizeof(T) == 2) r.v[0][i >> 1] |= i < c.have ? (uint32_t)__builtin_bit_cast(uint16_t, v) << (16 * (i & 1)) : 0u;
                else r.v[i >> 2][i & 3] = i < c.have ? __float_as_uint(v) : 0u;
            }
    }
    return r;
}
template <bool TAIL, class T> __device__ __forceinline__ void settle8(Raw8<T> &r, Cols c)
{
    if constexpr (TAIL)
        if (c.back) {
            constexpr int W = 2 * (int)sizeof(T);    // words
            uint32_t w[W];
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = r.v[i >> 2][i & 3];
            if (c.back & 4)
#pragma unroll
                for (int i = 0; i < W; ++i) w[i] = i + W / 2 < W ? w[i + W / 2] : 0u;
            if (c.back & 2)
#pragma unroll
                for (int i = 0; i < W; ++i) w[i] = i + W / 4 < W ? w[i + W / 4] : 0u;
            if (c.back & 1)
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const uint32_t next = i + 1 < W ? w[i + 1] : 0u;
                    w[i] = sizeof(T) == 4 ? next : __builtin_amdgcn_alignbit(next, w[i], 16);
                }
#pragma unroll
            for (int i = 0; i < W; ++i) r.v[i >> 2][i & 3] = w[i];
        }
}
// eight of a vector's values in 32 bits, or `otherwise` where there is none
template <bool TAIL, class T> __device__ __forceinline__ void vector8(float (&v)[8], const void *p, Cols c, float otherwise)
{
    if (p) {
        Raw8<T> r = raw8<TAIL>((const T *)p, c);
        settle8<TAIL>(r, c);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = r[i];
    } else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = otherwise;
}

// (mean, r) of a row that the lanes hold; v becomes (v - mean) r.  The variance is taken of the differences from the mean.
template <int LANES, int V>
__device__ __forceinline__ float2 normalise(float (&v)[V][8], const int (&have)[V], bool layer, float eps, float inv_n,
                                            RowSum<LANES> &sum)
{
    float mean = 0.0f;
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[j][i];        // (zeros beyond the row's end)
        mean = sum(s) * inv_n;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = i < have[j] ? v[j][i] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(v[j][i], v[j][i], s);
    const float r = 1.0f / sqrtf(fmaf(sum(s), inv_n, eps));
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] *= r;
    return {mean, r};
}

// Eight channels of each row a lane, LANES lanes a row.  F: there is an f; N: there is a next norm.  TAIL as in the backward
// kernel below: without one, lanes beyond the row's end go along with the first lane's channels, and no value needs a mask
// (16384 x 2048 with gate and dropout: 70 us with masks and sums through LDS, 58 without, 53.6 with the vectors' values in
// registers before anything waits).
template <class T, int LANES, bool F, bool N, bool TAIL>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) void block_fwd_kernel(Block a, T *y, T *h, float4 *stats)
{
    constexpr bool FAST = sizeof(T) == 2;
    constexpr int kThreads = LANES > 64 ? LANES : 256, kRows = kThreads / LANES;
    __shared__ float2 lds[2][RowSum<LANES>::kWaves];
    RowSum<LANES> sum(lds);
    const int lane = threadIdx.x % LANES;
    const bool live = lane * 8 < a.n;
    const Cols at = cols_of<TAIL>(lane, a.n);
    const int col = at.col, have = at.have;
    const bool drops = F && a.drop.below != 0;
    const DropKey key = drops ? drop_key(a.drop) : DropKey{};
    // (mean, r) of the values that the lanes hold, which become (v - mean) r; the variance is that of the differences
    auto normalise = [&](float (&v)[8], int kind) __attribute__((always_inline)) {
        float mean = 0.0f, s = 0.0f;
        if (kind == kNormLayer) {
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];            // (zeros beyond the row's end)
            mean = sum(TAIL || live ? s : 0.0f) * a.inv_n;
            s = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = !TAIL || i < have ? v[i] - mean : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
        const float r = 1.0f / sqrtf(fmaf(sum(TAIL || live ? s : 0.0f), a.inv_n, a.eps));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= r;
        return float2{mean, r};
    };
    // (the vectors' values for these channels, before anything waits)
    Raw8<T> w, b, scale, nw, nb;
    if constexpr (F) {
        if (a.w) w = raw8<TAIL>((const T *)a.w, at), settle8<TAIL>(w, at);
        if (a.b) b = raw8<TAIL>((const T *)a.b, at), settle8<TAIL>(b, at);
        if (a.scale) scale = raw8<TAIL>((const T *)a.scale, at), settle8<TAIL>(scale, at);
    }
    if constexpr (N) {
        if (a.nw) nw = raw8<TAIL>((const T *)a.nw, at), settle8<TAIL>(nw, at);
        if (a.nb) nb = raw8<TAIL>((const T *)a.nb, at), settle8<TAIL>(nb, at);
    }
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    if constexpr (LANES == 64) row = (int64_t)blockIdx.x * kRows + __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
    for (; row < a.m; row += (int64_t)gridDim.x * kRows) {
        float v[8];
        float4 st = {0.0f, 0.0f, 0.0f, 0.0f};
        Raw8<T> x = raw8<TAIL>((const T *)a.x + row * a.ldx, at);
        if constexpr (F) {
            Raw8<T> raw = raw8<TAIL>((const T *)a.f + row * a.ldf, at);
            Raw8<T> z;
            if (a.gate) z = raw8<TAIL>((const T *)a.gate + (int64_t)((uint32_t)row / (uint32_t)a.gate_div) * a.ldg, at);
            float f[8];
            settle8<TAIL>(raw, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = raw[i];
            if (a.norm != kNormNone) {
                const float2 s = normalise(f, a.norm);
                st.x = s.x;
                st.y = s.y;
                if (a.w)
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] *= w[i];
                if (a.b)
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] += b[i];
            }
            if (a.gate) {
                settle8<TAIL>(z, at);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= gate_of<FAST>(z[i], a.act);
            }
            if (a.scale)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= scale[i];
            if (drops) drop8(f, drop_numbers(key, (uint32_t)row, (uint32_t)col / 8), a.drop);
            settle8<TAIL>(x, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[i] + f[i];
            if (y && live) store8(y + row * a.n + col, v, have);
        } else {
            settle8<TAIL>(x, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = x[i];
        }
        if constexpr (N) {
            const float2 s = normalise(v, a.next);
            st.z = s.x;
            st.w = s.y;
            if (a.nw)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= nw[i];
            if (a.nb)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += nb[i];
            if (live) store8(h + row * a.n + col, v, have);
        }
        if (stats && lane == 0) stats[row] = st;
    }
}

// Rows of more than 8192 channels: V vectors of eight a lane.
template <class T, int LANES, int V, bool F, bool N>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) void block_fwd_long_kernel(Block a, T *y, T *h, float4 *stats)
{
    constexpr bool FAST = sizeof(T) == 2;
    constexpr int kThreads = LANES > 64 ? LANES : 256, kRows = kThreads / LANES;
    __shared__ float2 lds[2][RowSum<LANES>::kWaves];
    RowSum<LANES> sum(lds);
    const int lane = threadIdx.x % LANES;
    int col[V], have[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        col[j] = (j * LANES + lane) * 8;
        have[j] = max(0, min(8, a.n - col[j]));
    }
    const bool drops = F && a.drop.below != 0;
    const DropKey key = drops ? drop_key(a.drop) : DropKey{};
    const int64_t step = (int64_t)gridDim.x * kRows;
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES; row < a.m; row += step) {
        float v[V][8];
        float4 st = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < V; ++j) get8(v[j], (const T *)a.x + row * a.ldx + col[j], have[j]);
        if constexpr (F) {
            float f[V][8], p[8];
#pragma unroll
            for (int j = 0; j < V; ++j) get8(f[j], (const T *)a.f + row * a.ldf + col[j], have[j]);
            if (a.norm != kNormNone) {
                const float2 s = normalise<LANES, V>(f, have, a.norm == kNormLayer, a.eps, a.inv_n, sum);
                st.x = s.x;
                st.y = s.y;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (a.w) {
                        get8(p, (const T *)a.w + col[j], have[j]);
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[j][i] *= p[i];
                    }
                    if (a.b) {
                        get8(p, (const T *)a.b + col[j], have[j]);
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[j][i] += p[i];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (a.gate) {
                    get8(p, (const T *)a.gate + (int64_t)((uint32_t)row / (uint32_t)a.gate_div) * a.ldg + col[j], have[j]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[j][i] *= gate_of<FAST>(p[i], a.act);
                }
                if (a.scale) {
                    get8(p, (const T *)a.scale + col[j], have[j]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[j][i] *= p[i];
                }
                if (drops) drop8(f[j], drop_numbers(key, (uint32_t)row, (uint32_t)col[j] / 8), a.drop);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] += f[j][i];
                if (y) store8(y + row * a.n + col[j], v[j], have[j]);
            }
        }
        if constexpr (N) {
            const float2 s = normalise<LANES, V>(v, have, a.next == kNormLayer, a.eps, a.inv_n, sum);
            st.z = s.x;
            st.w = s.y;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float p[8];
                if (a.nw) {
                    get8(p, (const T *)a.nw + col[j], have[j]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[j][i] *= p[i];
                }
                if (a.nb) {
                    get8(p, (const T *)a.nb + col[j], have[j]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[j][i] += p[i];
                }
                store8(h + row * a.n + col[j], v[j], have[j]);
            }
        }
        if (stats && lane == 0) stats[row] = st;
    }
}

// ---- gradients
struct BlockGrads {
    const void *dy, *dh;
    const float4 *stats;
    void *dx, *df, *dgate;
    float2 *row_sums;        // [m] of the next norm, for the kernel that sums over rows by itself
    float *sums;             // [wanted ones][parts][n]: the vectors'; then [units][n], the gate's where its rows are cut
    uint32_t want;           // a bit each
    uint8_t slot[kSums];     // where the sums over rows lie in LDS (kNoSlot: not made), if they do
    int32_t parts;           // how many sums of a vector's there are: one a workgroup, of all its units
    Units units;
    __device__ __forceinline__ float *place(int k, int part, int n) const
    {
        return sums + ((int64_t)__popc(want & ((1u << k) - 1)) * parts + part) * n;
    }
};

// Of eight channels of a row: f normalised and w f^ + b.  Where a column is dropped, the gate and an f that no norm has taken in
// count as 0.
template <class T, bool F = true> struct Branch8 {
    static constexpr bool FAST = sizeof(T) == 2;
    const Block &a;
    const bool drops;
    const u32x4 numbers;
    const int64_t row;
    const int col, have;
    float fh[8], P[8];

    __device__ __forceinline__ Branch8(const Block &block, float4 st, bool d, u32x4 n, int64_t r, int c, int h)
        : a(block), drops(d), numbers(n), row(r), col(c), have(h)
    {
        if constexpr (!F) return;
        float p[8];
        get8(fh, (const T *)a.f + row * a.ldf + col, have);
        if (drops && a.norm == kNormNone) clear8(fh, numbers, a.drop);
#pragma unroll
        for (int i = 0; i < 8; ++i) P[i] = fh[i];
        if (a.norm != kNormNone) {
#pragma unroll
            for (int i = 0; i < 8; ++i) P[i] = fh[i] = i < have ? (fh[i] - st.x) * st.y : 0.0f;
            if (a.w) {
                get8(p, (const T *)a.w + col, have);
#pragma unroll
                for (int i = 0; i < 8; ++i) P[i] *= p[i];
            }
            if (a.b) {
                get8(p, (const T *)a.b + col, have);
#pragma unroll
                for (int i = 0; i < 8; ++i) P[i] += p[i];
            }
        }
    }
    __device__ __forceinline__ void gates(float (&z)[8]) const
    {
        get8(z, (const T *)a.gate + (int64_t)((uint32_t)row / (uint32_t)a.gate_div) * a.ldg + col, have);
        if (drops) clear8(z, numbers, a.drop);
    }
    // y += what the forward call added to x
    __device__ __forceinline__ void add_to(float (&y)[8]) const
    {
        float f[8], p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = P[i];
        if (a.gate) {
            gates(p);
            gate8<FAST>(p, a.act);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= p[i];
        }
        if (a.scale) {
            get8(p, (const T *)a.scale + col, have);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= p[i];
        }
        if (drops) drop8(f, numbers, a.drop);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += f[i];
    }
    // From the gradient d of y: dP, and what goes to dscale and dgate.
    __device__ __forceinline__ void terms(float (&d)[8], float (&dscale)[8], float (&dgate)[8]) const
    {
        float s[8];
        if (drops) drop8(d, numbers, a.drop);
        load_or<T>(s, a.scale, col, have, 1.0f);
        if (a.gate) {
            float z[8];
            gates(z);
#pragma unroll
            for (int i = 0; i < 8; ++i) dgate[i] = d[i] * s[i] * P[i];
            gate8<FAST>(z, dgate, a.act);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= z[i];
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) dgate[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dscale[i] = d[i] * P[i];
            d[i] *= s[i];
        }
    }
};

// The next norm's part in a row's gradients: t = dh w, y normalised, g = dh.  add: of y from x, where that is to be done.
template <class T, bool F, class Add>
__device__ __forceinline__ void next_norm_terms(float (&t)[8], float (&yh)[8], float (&g)[8], const Block &a, const BlockGrads &o,
                                                float4 st, int64_t row, int col, int have, Add add)
{
    float p[8];
    get8(g, (const T *)o.dh + row * a.n + col, have);
    get8(yh, (const T *)a.x + row * a.ldx + col, have);
    if constexpr (F && sizeof(T) == 2)
        if (a.again) add(yh);
    load_or<T>(p, a.nw, col, have, 1.0f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        yh[i] = (yh[i] - st.z) * st.w;
        t[i] = g[i] * p[i];
    }
}

// A lane has the same eight channels of every row of its unit.  Up to 4096 channels (SLOTS 0) it has the vectors' values for
// them and their sums over the rows in registers, with the next row's values on their way while it works on one.  With more
// (1024 lanes, 128 registers each) the sums lie in LDS, a slot of 8192 floats each, where a lane meets nobody else's, the vectors are
// read again for every row, and only rows in bf16 come ahead of time.  Without a TAIL the channels are a multiple
// of eight: a lane has eight or none, and one that has none goes along with the first lane's (in bounds, left out of
// the row's sums and not stored).
//
// y in bf16 was rounded, and h is not made of that: y is made again of x and f, the same bytes and a tenth more instructions
// (16384 x 2048 with gate and dropout, forward and gradients, 149 -> 152 us, 4096 x 8192 with norms and scale 168 -> 177; the
// gradients of the next norm are off by bf16's rounding of themselves, 1.7e-3 of their norm, where a rounded y makes that 2.3e-3, and
// anything where y's mean is large beside what a layer norm is made of).
//
// What dropout has taken out has no part in any gradient, whatever it was: beside a gradient of 0 the gate, and f where no norm takes
// in its row, count as 0 (1 % of the time).
//
// Which norm and gate is asked once for a row's eight channels, not for each (4096 x 4096 in f32 with layer norms, a sigmoid gate and
// dropout, both ways, 195 -> 175 us); what is the same in all lanes of a wave lies in scalar registers.
//
// With s = t act(gate), A = sum s (f - mu) r and B = sum s two sums over rows give three gradients:
// dscale = w A + b B, dweight = scale A, dbias = scale B.
//
// Three waves to a SIMD, as the registers allow: 768 workgroups of 256 lanes (16384 x 2048: 92 us; 1024 workgroups without the
// next row on its way, a third of them in a second round, masks at every value and sums by LDS permutes: 220).  4096 rows of 8192
// channels 107 us, with the sums in LDS; 260 and more in two passes.
template <class T, int LANES, bool F, bool N, bool TAIL, int SLOTS>
__global__ __launch_bounds__(LANES > 64 ? LANES : 64) void block_bwd_kernel(Block a, BlockGrads o)
{
    constexpr bool FAST = sizeof(T) == 2, WIDE = SLOTS > 0, AHEAD = !WIDE || sizeof(T) == 2, AGAIN = F && N && sizeof(T) == 2;
    __shared__ float2 lds[2][RowSum<LANES>::kWaves];
    __shared__ f32x4 slots[WIDE ? SLOTS : 1][2][WIDE ? LANES : 1];
    RowSum<LANES> sum(lds);
    const int lane = threadIdx.x % LANES;
    const bool live = lane * 8 < a.n;
    const Cols at = cols_of<TAIL>(lane, a.n);
    const int col = at.col, have = at.have;
    constexpr int kUnits = LANES > 64 ? 1 : 64 / LANES;
    int unit = (int)blockIdx.x * kUnits + (LANES > 64 ? 0 : threadIdx.x / LANES);
    if constexpr (LANES == 64) unit = __builtin_amdgcn_readfirstlane(unit);
    int64_t row = 0, end = 0;                        // (a wave's last lanes may be without a unit)
    if (unit < o.units.count) range_of(o.units, unit, a.m, row, end);
    const bool drops = F && a.drop.below != 0, next = N && o.dh, normed = F && a.norm != kNormNone;
    const bool own_gates = F && o.dgate && a.gate_div == 1, whole_gates = F && o.dgate && a.gate_div > 1 && o.units.cuts == 1;
    const DropKey key = drops ? drop_key(a.drop) : DropKey{};

    // the vectors: once, or where they are used; of the branch, w and b times scale and what dropout multiplies by
    constexpr int kOnce = WIDE ? 1 : 8;
    const float factor = drops ? a.drop.factor : 1.0f;
    float nw_[kOnce], ws_[kOnce], bs_[kOnce];
    auto scaled = [&](float (&ws)[8], float (&bs)[8]) __attribute__((always_inline)) {
        float s[8];
        vector8<TAIL, T>(s, a.scale, at, 1.0f);
        vector8<TAIL, T>(ws, a.w, at, 1.0f);
        vector8<TAIL, T>(bs, a.b, at, 0.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] *= factor;
            ws[i] *= s[i];
            if (a.b) bs[i] *= s[i];
        }
    };
    if constexpr (!WIDE) {
        if constexpr (N) vector8<TAIL, T>(nw_, a.nw, at, 1.0f);
        if constexpr (F) scaled(ws_, bs_);
    }
    auto kept_or = [&](float (&v)[8], const float (&once)[kOnce]) __attribute__((always_inline)) {
        if constexpr (!WIDE)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = once[i];
    };
    // the sums over the rows: step(i, sum so far) for each channel
    float sums_[WIDE ? 1 : kSums][8];
    auto sum_of = [&](int k, auto step) __attribute__((always_inline)) {
        if constexpr (WIDE) {
            if (o.slot[k] < SLOTS) {
                f32x4 v[2] = {slots[o.slot[k]][0][lane], slots[o.slot[k]][1][lane]};
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i >> 2][i & 3] = step(i, v[i >> 2][i & 3]);
                slots[o.slot[k]][0][lane] = v[0];
                slots[o.slot[k]][1][lane] = v[1];
            }
        } else
#pragma unroll
            for (int i = 0; i < 8; ++i) sums_[k][i] = step(i, sums_[k][i]);
    };
    auto take = [&](int k, float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        sum_of(k, [&](int i, float s) __attribute__((always_inline)) { v[i] = s; return s; });
    };
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        if constexpr (WIDE) sum_of(k, [](int, float) __attribute__((always_inline)) { return 0.0f; });
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) sums_[k][i] = 0.0f;
    }

    struct Row {
        Raw8<T> dy, dh, y, f, z;
        float4 st;
    };
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {
        Row v;
        if (o.stats) v.st = o.stats[r];
        else v.st = float4{0.0f, 1.0f, 0.0f, 1.0f};
        if (o.dy) v.dy = raw8<TAIL>((const T *)o.dy + r * a.n, at);
        if (next) {
            v.dh = raw8<TAIL>((const T *)o.dh + r * a.n, at);
            v.y = raw8<TAIL>((const T *)a.x + r * a.ldx, at);
        }
        if constexpr (F) {
            v.f = raw8<TAIL>((const T *)a.f + r * a.ldf, at);
            if (a.gate) v.z = raw8<TAIL>((const T *)a.gate + (int64_t)((uint32_t)r / (uint32_t)a.gate_div) * a.ldg, at);
        }
        return v;
    };
    Row ahead;
    if constexpr (AHEAD)
        if (row < end) ahead = fetch(row);
    for (; row < end; ++row) {
        Row v;
        if constexpr (AHEAD) {
            v = ahead;
            if (row + 1 < end) ahead = fetch(row + 1);
        } else v = fetch(row);
        if constexpr (LANES >= 64) v.st = float4{of_wave(v.st.x), of_wave(v.st.y), of_wave(v.st.z), of_wave(v.st.w)};
        if (o.dy) settle8<TAIL>(v.dy, at);
        float d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = o.dy ? v.dy[i] : 0.0f;
        // f normalised, w scale times dropout's factor, and d scale (w f^ + b), d dropout's factor or 0
        float fh[8], ws[8], e[8];
        const float mu = normed && a.norm == kNormLayer ? v.st.x : 0.0f, r = normed ? v.st.y : 1.0f;
        u32x4 numbers;
        auto branch = [&](bool whole) __attribute__((always_inline)) {
            float bs[8];
            if constexpr (WIDE) scaled(ws, bs);
            kept_or(ws, ws_);
            kept_or(bs, bs_);
#pragma unroll
            for (int i = 0; i < 8; ++i) fh[i] = (v.f[i] - mu) * r;
            if (drops && !normed) clear8(fh, numbers, a.drop);       // (a norm takes in the whole row)
            if (whole) {
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = fmaf(fh[i], ws[i], bs[i]);
                if (drops) clear8(e, numbers, a.drop);
            }
        };
        auto gates = [&](float (&z)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = v.z[i];
            if (drops) clear8(z, numbers, a.drop);
        };
        if constexpr (F) {
            if (drops) numbers = drop_numbers(key, (uint32_t)row, (uint32_t)col / 8);
            settle8<TAIL>(v.f, at);
            if (a.gate) settle8<TAIL>(v.z, at);
            if constexpr (AGAIN) branch(a.gate || (next && a.again));
        }
        if (next) {
            float t[8], yh[8], s1 = 0.0f, s2 = 0.0f;
            settle8<TAIL>(v.dh, at);
            settle8<TAIL>(v.y, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) yh[i] = v.y[i];
            if constexpr (AGAIN)
                if (a.again) {
                    if (a.gate) {
                        float z[8];
                        gates(z);
                        gate8<FAST>(z, a.act);
#pragma unroll
                        for (int i = 0; i < 8; ++i) yh[i] = fmaf(e[i], z[i], yh[i]);
                    } else
#pragma unroll
                        for (int i = 0; i < 8; ++i) yh[i] += e[i];
                }
            if constexpr (WIDE) vector8<TAIL, T>(t, a.nw, at, 1.0f);
            kept_or(t, nw_);
            const float next_mu = a.next == kNormLayer ? v.st.z : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                yh[i] = (yh[i] - next_mu) * v.st.w;
                t[i] *= v.dh[i];
                s1 += t[i];
                s2 = fmaf(t[i], yh[i], s2);
            }
            sum_of(kSumDnw, [&](int i, float s) __attribute__((always_inline)) { return fmaf(v.dh[i], yh[i], s); });
            sum_of(kSumDnb, [&](int i, float s) __attribute__((always_inline)) { return s + v.dh[i]; });
            if (!TAIL && !live) s1 = s2 = 0.0f;
            const float2 c = sum(s1, s2);
            const float k1 = a.next == kNormLayer ? -v.st.w * c.x * a.inv_n : 0.0f, k2 = -v.st.w * c.y * a.inv_n;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] += fmaf(v.st.w, t[i], fmaf(yh[i], k2, k1));
                if (TAIL && i >= have) d[i] = 0.0f;
            }
        }
        if (o.dx && live) store8((T *)o.dx + row * a.n + col, d, have);
        if constexpr (F) {
            float s1 = 0.0f, s2 = 0.0f;
            if constexpr (!AGAIN || WIDE) branch(a.gate);   // (wide: once more, in place of registers that there are not)
            if (drops) clear8(d, numbers, a.drop);
            if (a.gate) {
                float dg[8], z[8];
                gates(z);
#pragma unroll
                for (int i = 0; i < 8; ++i) dg[i] = d[i] * e[i];
                gate8<FAST>(z, dg, a.act);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= z[i];
                sum_of(kSumGate, [&](int i, float s) __attribute__((always_inline)) { return s + dg[i]; });
                if (own_gates && live) store8((T *)o.dgate + row * a.n + col, dg, have);
                if (whole_gates && ((uint32_t)row + 1) % (uint32_t)a.gate_div == 0) {
                    take(kSumGate, dg);
                    if (live) store8((T *)o.dgate + (int64_t)((uint32_t)row / (uint32_t)a.gate_div) * a.n + col, dg, have);
                    sum_of(kSumGate, [](int, float) __attribute__((always_inline)) { return 0.0f; });
                }
            }
            sum_of(kSumA, [&](int i, float s) __attribute__((always_inline)) { return fmaf(d[i], fh[i], s); });
            sum_of(kSumB, [&](int i, float s) __attribute__((always_inline)) { return s + d[i]; });
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= ws[i];
            if (normed) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s1 += d[i];
                    s2 = fmaf(d[i], fh[i], s2);
                }
                if (!TAIL && !live) s1 = s2 = 0.0f;
                const float2 c = sum(s1, s2);
                const float k1 = a.norm == kNormLayer ? -v.st.y * c.x * a.inv_n : 0.0f, k2 = -v.st.y * c.y * a.inv_n;
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = fmaf(v.st.y, d[i], fmaf(fh[i], k2, k1));
            }
            if (o.df && live) store8((T *)o.df + row * a.n + col, d, have);
        }
    }
    // a workgroup's sums leave together: those of a wave's units are joined in it (a cut gate's are not, they stay apart)
    auto joined = [&](int k, float (&v)[8]) __attribute__((always_inline)) {
        take(k, v);
#pragma unroll
        for (int j = LANES; j < 64; j <<= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += __shfl_xor(v[i], j);
    };
    auto leave = [&](int k, const float (&v)[8]) __attribute__((always_inline)) {
        if (live && threadIdx.x < LANES && (o.want >> k & 1)) store8(o.place(k, blockIdx.x, a.n) + col, v, have);
    };
    float v[8];
    if constexpr (F) {
        float A[8], B[8], w[8], b[8], scale[8];
        joined(kSumA, A);
        joined(kSumB, B);
        vector8<TAIL, T>(w, a.w, at, 1.0f);
        vector8<TAIL, T>(b, a.b, at, 0.0f);
        vector8<TAIL, T>(scale, a.scale, at, 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) A[i] *= factor, B[i] *= factor;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = scale[i] * A[i];
        leave(kDw, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = scale[i] * B[i];
        leave(kDb, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(w[i], A[i], b[i] * B[i]);
        leave(kDscale, v);
        take(kSumGate, v);
        if (live && unit < o.units.count && (o.want >> kVectors & 1)) store8(o.place(kVectors, unit, a.n) + col, v, have);
    }
    joined(kSumDnw, v);
    leave(kDnw, v);
    joined(kSumDnb, v);
    leave(kDnb, v);
}

// Rows of more channels: one row after the other, without sums over them.
template <class T, int LANES, int V, bool F, bool N>
__global__ __launch_bounds__(LANES) void block_rows_kernel(Block a, BlockGrads o)
{
    __shared__ float2 lds[2][RowSum<LANES>::kWaves];
    RowSum<LANES> sum(lds);
    const int lane = threadIdx.x % LANES;
    int col[V], have[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        col[j] = (j * LANES + lane) * 8;
        have[j] = max(0, min(8, a.n - col[j]));
    }
    const bool drops = F && a.drop.below != 0;
    const DropKey key = drops ? drop_key(a.drop) : DropKey{};
    const bool next = N && o.dh;
    for (int64_t row = blockIdx.x; row < a.m; row += gridDim.x) {
        const float4 st = (N || F) && o.stats ? o.stats[row] : float4{0.0f, 1.0f, 0.0f, 1.0f};
        float d[V][8];
        u32x4 numbers[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            numbers[j] = drops ? drop_numbers(key, (uint32_t)row, (uint32_t)col[j] / 8) : u32x4{0, 0, 0, 0};
            if (o.dy) get8(d[j], (const T *)o.dy + row * a.n + col[j], have[j]);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) d[j][i] = 0.0f;
        }
        if constexpr (N) {
            if (next) {
                float t[V][8], yh[V][8], g[8], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    next_norm_terms<T, F>(t[j], yh[j], g, a, o, st, row, col[j], have[j], [&](float (&y)[8]) __attribute__((always_inline)) {
                        Branch8<T>(a, st, drops, numbers[j], row, col[j], have[j]).add_to(y);
                    });
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        s1 += t[j][i];
                        s2 = fmaf(t[j][i], yh[j][i], s2);
                    }
                }
                float2 c = sum(s1, s2);
                c.x = a.next == kNormLayer ? c.x * a.inv_n : 0.0f;
                c.y *= a.inv_n;
                if (o.row_sums && lane == 0) o.row_sums[row] = c;
#pragma unroll
                for (int j = 0; j < V; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        d[j][i] = i < have[j] ? fmaf(st.w, t[j][i] - c.x - yh[j][i] * c.y, d[j][i]) : 0.0f;
            }
        }
        if (o.dx)
#pragma unroll
            for (int j = 0; j < V; ++j) store8((T *)o.dx + row * a.n + col[j], d[j], have[j]);
        if constexpr (F) {
            float fh[V][8], dscale[8], dgate[8], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                // (once more, in place of registers that there are not)
                const Branch8<T> branch(a, st, drops, numbers[j], row, col[j], have[j]);
                branch.terms(d[j], dscale, dgate);
#pragma unroll
                for (int i = 0; i < 8; ++i) fh[j][i] = branch.fh[i];
                if (o.dgate && a.gate_div == 1) store8((T *)o.dgate + row * a.n + col[j], dgate, have[j]);
                if (a.norm != kNormNone) {
                    float p[8];
                    load_or<T>(p, a.w, col[j], have[j], 1.0f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        d[j][i] *= p[i];
                        s1 += d[j][i];
                        s2 = fmaf(d[j][i], fh[j][i], s2);
                    }
                }
            }
            if (a.norm != kNormNone) {
                float2 c = sum(s1, s2);
                c.x = a.norm == kNormLayer ? c.x * a.inv_n : 0.0f;
                c.y *= a.inv_n;
#pragma unroll
                for (int j = 0; j < V; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[j][i] = st.y * (d[j][i] - c.x - fh[j][i] * c.y);
            }
            if (o.df)
#pragma unroll
                for (int j = 0; j < V; ++j) store8((T *)o.df + row * a.n + col[j], d[j], have[j]);
        }
    }
}

// The sums over rows where a row has more channels than its lanes could keep sums of: a lane has eight channels of a run of
// rows, and takes each row's own sums (its gradient's mean and the like) from the kernel above.
template <class T, bool F, bool N>
__global__ __launch_bounds__(256) void block_sums_kernel(Block a, BlockGrads o)
{
    const int col = ((int)blockIdx.x * 256 + threadIdx.x) * 8, have = max(0, min(8, a.n - col)), unit = blockIdx.y;
    if (have == 0) return;
    const bool drops = F && a.drop.below != 0;
    const DropKey key = drops ? drop_key(a.drop) : DropKey{};
    int64_t row, end;
    range_of(o.units, unit, a.m, row, end);
    float acc[kVectors + 1][8];
#pragma unroll
    for (int k = 0; k <= kVectors; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[k][i] = 0.0f;
    for (; row < end; ++row) {
        const float4 st = o.stats ? o.stats[row] : float4{0.0f, 1.0f, 0.0f, 1.0f};
        const u32x4 numbers = drops ? drop_numbers(key, (uint32_t)row, (uint32_t)col / 8) : u32x4{0, 0, 0, 0};
        const Branch8<T, F> branch(a, st, drops, numbers, row, col, have);
        float d[8];
        if (o.dy) get8(d, (const T *)o.dy + row * a.n + col, have);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = 0.0f;
        if constexpr (N)
            if (o.dh) {
                float t[8], yh[8], g[8];
                next_norm_terms<T, F>(t, yh, g, a, o, st, row, col, have,
                                      [&](float (&y)[8]) __attribute__((always_inline)) { branch.add_to(y); });
                const float2 c = o.row_sums[row];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    acc[kDnw][i] = fmaf(g[i], yh[i], acc[kDnw][i]);
                    acc[kDnb][i] += g[i];
                    d[i] = i < have ? fmaf(st.w, t[i] - c.x - yh[i] * c.y, d[i]) : 0.0f;
                }
            }
        if constexpr (F) {
            float dscale[8], dgate[8];
            branch.terms(d, dscale, dgate);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc[kDscale][i] += dscale[i];
                acc[kVectors][i] += dgate[i];
                acc[kDw][i] = fmaf(d[i], branch.fh[i], acc[kDw][i]);
                acc[kDb][i] += d[i];
            }
            if (o.dgate && a.gate_div > 1 && o.units.cuts == 1 && ((uint32_t)row + 1) % (uint32_t)a.gate_div == 0) {
                store8((T *)o.dgate + (int64_t)((uint32_t)row / (uint32_t)a.gate_div) * a.n + col, acc[kVectors], have);
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[kVectors][i] = 0.0f;
            }
        }
    }
#pragma unroll
    for (int k = 0; k <= kVectors; ++k)
        if (o.want >> k & 1) store8(o.place(k, unit, a.n) + col, acc[k], have);
}

// The units' sums, joined in their order: workgroup (columns, y) has the y-th wanted sum.  Bound by the latency of its loads:
// 32 of a column's parts at a time 4.8 us for 745 parts of 2048 channels, eight at a time 7.5.
struct Joins {
    const float *from[kVectors];
    void *to[kVectors];
    const float *gate_from;
    void *gate_to;
    int32_t vectors, parts, cuts, n;
};
template <class T> __global__ __launch_bounds__(1024) void block_join_kernel(Joins j)
{
    constexpr int kGroups = 32;
    __shared__ float part[kGroups][32];
    const int c = threadIdx.x & 31, g = threadIdx.x >> 5, col = (int)blockIdx.x * 32 + c, y = blockIdx.y;
    const float *from = y < j.vectors ? j.from[y] : j.gate_from + (int64_t)(y - j.vectors) * j.cuts * j.n;
    T *to = y < j.vectors ? (T *)j.to[y] : (T *)j.gate_to + (int64_t)(y - j.vectors) * j.n;
    const int count = y < j.vectors ? j.parts : j.cuts;
    float s = 0.0f;
    if (col < j.n)
#pragma unroll 8
        for (int u = g; u < count; u += kGroups) s += from[(int64_t)u * j.n + col];
    part[g][c] = s;
    __syncthreads();
    if (g == 0 && col < j.n) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) s += part[i][c];
        to[col] = narrow<T>(s);
    }
}

}  // namespace tvl
