// Checks the backward call's plan of residual borders for each set of operands and wanted gradients, a size a line of the input:
// m n shared gate_div.  Prints a line a size: "ok" and how many plans it looked at, or what is wrong.
#include "../paper_2204_03643_amd/csrc/tv_block_plan.hpp"
#include <cstdio>

using namespace tvl;

static const char *plan_wrong(const tv_block_in &in, const tv_block_grads &g, const tv_block_desc &d)
{
    const BlockBwdPlan p = block_bwd_plan(in, g, d);
    const bool shared = in.f && in.gate && g.dgate && d.gate_div > 1, cut = shared && p.units.cuts > 1;
    const void *wanted[kVectors] = {in.f ? g.dweight : nullptr, in.f ? g.dbias : nullptr, in.f ? g.dscale : nullptr, g.dnext_weight, g.dnext_bias};
    int64_t vectors = 0;
    for (int k = 0; k < kVectors; ++k) {
        if ((p.want >> k & 1) != (wanted[k] != nullptr)) return "a vector's bit is wrong";
        vectors += wanted[k] != nullptr;
    }
    if ((p.want >> kVectors & 1) != cut) return "the gate's bit is wrong";
    // a workgroup's sums of each vector, and each unit's of a gate that is cut, side by side
    const size_t sums = (size_t)(vectors * p.parts + (cut ? p.units.count : 0)) * d.n * 4;
    if (p.row_sums < sums || p.row_sums % 16 || p.bytes < p.row_sums) return "a workspace that is too small";
    if (block_lanes(d.n) <= kMostSumLanes) return p.two_passes || p.slots ? "slots or passes without need" : nullptr;
    if (p.two_passes) return (p.want || shared) && p.bytes < p.row_sums + (size_t)d.m * 8 ? "no place for the rows' sums" : nullptr;
    if (p.slots > kMostSlots || d.n > 8192) return "more sums than fit";
    // the sums that each gradient is made of have slots of their own
    const bool bias = in.bias && d.norm != TV_NORM_NONE;
    const bool made[kSums] = {in.f && (g.dweight || g.dscale), in.f && (g.dbias || (g.dscale && bias)), g.dnext_weight != nullptr,
                              g.dnext_bias != nullptr, shared};
    unsigned met = 0;
    for (int k = 0; k < kSums; ++k) {
        if (!made[k]) {
            if (p.slot[k] != kNoSlot) return "a slot for nothing";
            continue;
        }
        if (p.slot[k] >= p.slots) return "a sum without a slot";
        if (met >> p.slot[k] & 1) return "two sums in a slot";
        met |= 1u << p.slot[k];
    }
    return nullptr;
}

int main()
{
    long long m, n, shared, div;
    while (scanf("%lld %lld %lld %lld", &m, &n, &shared, &div) == 4) {
        char there;
        const char *wrong = nullptr;
        int looked = 0;
        for (int bits = 0; bits < 1 << 11 && !wrong; ++bits) {
            auto bit = [&](int k) { return bits >> k & 1 ? &there : nullptr; };
            tv_block_in in{};
            tv_block_grads g{};
            tv_block_desc d{};
            in.x = &there;
            in.f = bit(0); in.bias = bit(1); in.gate = shared ? &there : nullptr;
            g.dx = bit(2); g.df = bit(3); g.dweight = bit(4); g.dbias = bit(5); g.dscale = bit(6); g.dgate = bit(7);
            g.dnext_weight = bit(8); g.dnext_bias = bit(9);
            d.norm = bits >> 10 & 1 ? TV_NORM_LAYER : TV_NORM_NONE;
            d.next_norm = TV_NORM_RMS;
            d.m = m; d.n = n; d.gate_div = shared ? div : 1;
            // what the call refuses
            if (!in.f && (g.df || g.dgate || g.dweight || g.dbias || g.dscale)) continue;
            if ((g.dgate && !in.gate) || (d.norm == TV_NORM_NONE && (g.dweight || g.dbias))) continue;
            wrong = plan_wrong(in, g, d);
            ++looked;
        }
        if (wrong) printf("%s\n", wrong);
        else printf("ok %d\n", looked);
    }
    return 0;
}
