// How the rows of a residual border are shared out and how the backward call's workspace is laid out.  Host code alone: it
// needs no GPU compiler.
#pragma once
#include "tv_linear_plan.hpp"

namespace tvl {

constexpr int kVectors = 5;                  // sums over rows, in this order; the gate's are the sixth
enum Vector : int { kDw = 0, kDb = 1, kDscale = 2, kDnw = 3, kDnb = 4 };
constexpr int kSums = 5;                     // what is summed over rows to make them: see block_bwd_kernel
enum Sum : int { kSumA = 0, kSumB = 1, kSumDnw = 2, kSumDnb = 3, kSumGate = 4 };
constexpr int kNoSlot = 255, kMostSlots = 4; // of 8192 floats each in LDS

// Lanes side by side in a row of n channels, eight channels each (twice eight from 8193 channels on).
inline int block_lanes(int64_t n)
{
    const int64_t per = tiles(n, 8);
    for (int lanes : {8, 16, 32, 64, 128, 256, 512})
        if (per <= lanes) return lanes;
    return 1024;
}
constexpr int kMostSumLanes = 512;           // with more, lanes keep no sums over rows in registers

// Units are runs of rows whose sums one group of lanes makes.  A gate's rows that are shared by several rows of x are either
// cut into `cuts` units each, whose sums are joined afterwards, or lie whole within a unit (cuts 1).
struct Units {
    int64_t span;            // rows that a gate's row stands for (cuts > 1), or all rows
    int32_t rows, cuts, per; // rows of a unit; units a gate's row; units a span
    int32_t count;
};

// The rows of a unit.
#ifdef __HIPCC__
__host__ __device__
#endif
inline void range_of(const Units &u, int unit, int64_t m, int64_t &begin, int64_t &end)
{
    const int64_t first = unit / u.per * u.span, last = first + u.span < m ? first + u.span : m;
    begin = first + (int64_t)(unit % u.per) * u.rows;
    end = begin + u.rows < last ? begin + u.rows : last;
}

// As many units as fill the card three waves to a SIMD deep, two rows at least from 513 rows on (every unit writes its sums
// once: a row each would cost more bytes than the row has).
inline Units block_units(int64_t m, int64_t n, bool shared_gate, int64_t gate_div)
{
    const int lanes = block_lanes(n);
    const int64_t most = lanes > kMostSumLanes ? 256 : 256 * 768 / lanes;
    int64_t rows = tiles(m, most);
    if (rows < 2) rows = m > 512 ? 2 : 1;
    Units u{m, 0, 1, 0, 0};
    if (shared_gate && gate_div > rows) {
        u.cuts = (int32_t)tiles(gate_div, rows);
        rows = tiles(gate_div, u.cuts);
        u.cuts = (int32_t)tiles(gate_div, rows);
        u.span = gate_div;
        u.per = u.cuts;
        u.count = m > 0 ? (int32_t)(m / gate_div * u.cuts) : 0;
    } else {
        if (shared_gate) rows = rows / gate_div * gate_div;
        u.per = u.count = (int32_t)tiles(m, rows);
    }
    u.rows = (int32_t)rows;
    return u;
}

struct BlockBwdPlan {
    Units units;
    int32_t parts;           // workgroups, each with sums of its units
    uint32_t want;           // a bit a vector, and the gate's where its rows are cut
    int slots;               // sums over rows in LDS; 0: in registers
    uint8_t slot[kSums];
    bool two_passes;         // the rows first, the sums over them in a pass of their own
    size_t row_sums, bytes;  // where the rows' own sums lie
};

inline BlockBwdPlan block_bwd_plan(const tv_block_in &in, const tv_block_grads &g, const tv_block_desc &d)
{
    BlockBwdPlan p{};
    const bool shared = in.f && in.gate && g.dgate && d.gate_div > 1;
    p.units = block_units(d.m, d.n, shared, d.gate_div);
    const void *vectors[kVectors] = {in.f ? g.dweight : nullptr, in.f ? g.dbias : nullptr, in.f ? g.dscale : nullptr, g.dnext_weight, g.dnext_bias};
    p.parts = (int32_t)(block_lanes(d.n) < 64 ? tiles(p.units.count, 64 / block_lanes(d.n)) : p.units.count);
    int64_t wanted = 0;
    for (int k = 0; k < kVectors; ++k)
        if (vectors[k]) p.want |= 1u << k, ++wanted;
    const bool cut = shared && p.units.cuts > 1;
    if (cut) p.want |= 1u << kVectors;
    p.row_sums = (size_t)up((wanted * p.parts + (cut ? p.units.count : 0)) * d.n * 4, 256);
    p.bytes = p.row_sums;
    if (block_lanes(d.n) > kMostSumLanes) {
        // Sums in LDS where its slots are enough: up to 8192 channels, and all but both norms' biases beside a shared gate
        // (4096 rows of 8192 bf16 channels, two norms and a scale: 107 us, and more than 260 in two passes).
        const bool bias = in.bias && d.norm != TV_NORM_NONE;
        const bool made[kSums] = {in.f && (g.dweight || g.dscale), in.f && (g.dbias || (g.dscale && bias)), g.dnext_weight != nullptr,
                                  g.dnext_bias != nullptr, shared};
        for (int k = 0; k < kSums; ++k) p.slot[k] = made[k] ? (uint8_t)p.slots++ : (uint8_t)kNoSlot;
        p.two_passes = p.slots > kMostSlots || d.n > 8192;
        if (p.two_passes && (p.want || shared)) p.bytes += (size_t)up(d.m * 8, 256);
    }
    return p;
}

}  // namespace tvl
