// Which kernels a product in 4 bits takes, how its contraction is split and how its workspace is laid out.  Host code alone:
// it needs no GPU compiler.
#pragma once
#include "tv_linear_plan.hpp"

namespace tvl {

constexpr int64_t kMostGroups4 = TV_LINEAR4_MAX_K / TV_MX4_GROUP;       // so that a tile's rows span less than 2^32 bytes

inline int64_t groups_of(int64_t n) { return tiles(n, TV_MX4_GROUP); }
inline int64_t scale_rows(int64_t rows) { return up(rows, 4); }

// How a call goes.  kFew4: the weight streamed through registers, x taken to 4 bits by each workgroup (own) or before.
enum Kind4 { kFew4, kTile64x4, kTile128x4, kTile256x4 };
struct Choice4 {
    Kind4 kind;
    bool own;
    int splits, k_per;       // contraction in 32 a group
    double us;
};

inline Choice4 cut4(Kind4 kind, bool own, int64_t s, int64_t groups, int64_t unit)
{
    const int64_t per = up(tiles(groups, s < 1 ? 1 : s), unit);
    return {kind, own, (int)tiles(groups, per), (int)per * 32, 0.0};
}

constexpr int64_t kFewRows4 = 32, kOwnValues4 = 16384, kOwnLength4 = 8192;

// Sizes alone decide.  Up to 32 rows stream the weight (2048 -> 8192, x taken to 4 bits included: 32 rows 7.6 us streamed, 8.1
// through tiles; 64 rows 9.8 and 8.4), few values of x in the same launch (one row of 2048 -> 8192 5.1 us in one, 6.2 in two; 16 rows,
// 32768 values, 7.5 and 6.6; one row of 8192 -> 2048 8.3 and 7.9, of 16384 -> 4096 16.1 and 13.1).  Otherwise the cheapest by a model of the time in microseconds, fitted to
// sweeps of tiles and splits over outputs of 64 x 1024 to 8192 x 8192 and contractions of 1024 to 8192: a launch; rounds of
// workgroups over 256 compute units, in each a start and an end and so much a step of 256; for split contractions the second launch
// and the sums' trip through memory.
inline Choice4 choose4(bool codes, int64_t M, int64_t N, int64_t K, int64_t groups)
{
    // (as long as a launch of 512 threads for every 16 columns has fewer than 2^32)
    if (M <= kFewRows4 && N <= ((int64_t)1 << 26)) return cut4(kFew4, !codes && M <= 16 && K <= kOwnLength4 && M * K <= kOwnValues4, 1, groups, 8);
    struct Cost { Kind4 kind; int m, n; double round, step; };
    constexpr Cost costs[] = {{kTile64x4, 64, 128, 1.5, 0.30}, {kTile128x4, 128, 128, 2.4, 0.60}, {kTile256x4, 256, 256, 6.0, 1.75}};
    Choice4 best{};
    best.us = 1e30;
    for (const Cost &c : costs) {
        const int64_t t = tiles(M, c.m) * tiles(N, c.n);
        for (int s : {1, 2, 3, 4, 6, 8}) {
            if (s > 1 && (groups < 4 * s || t * s > 1024)) break;
            Choice4 x = cut4(c.kind, false, s, groups, 2);
            x.us = 3.0 + (double)tiles(t * x.splits, 256) * (c.round + c.step * (double)tiles(x.k_per, 64));
            if (x.splits > 1) x.us += 2.6 + 0.18 * x.splits + (double)M * (double)N * x.splits * 8 / 7e6;
            if (x.us < best.us) best = x;
        }
    }
    return best;
}

// The workspace: x's codes and scale words (where they are made before), split sums.
struct Plan4 {
    Choice4 c;
    size_t exps, split, bytes;
};

inline Plan4 plan4(const tv_linear_desc &d, bool codes)
{
    Plan4 p{};
    p.c = choose4(codes, d.m, d.n, d.k, groups_of(d.k));
    if (!codes && !p.c.own) {
        p.exps = (size_t)up(d.m * groups_of(d.k) * 64, 256);
        p.split = p.exps + (size_t)up(scale_rows(d.m) * groups_of(d.k) * 4, 256);
    }
    p.bytes = p.split + (p.c.splits > 1 ? (size_t)up((int64_t)p.c.splits * d.m * up(d.n, 8) * 4, 256) : 0);
    return p;
}

}  // namespace tvl
