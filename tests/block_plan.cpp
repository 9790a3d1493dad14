// Checks how the rows of residual borders are shared out, a call a line of the input: m n shared gate_div; and, after a line
// of zeros, the launches of products in 4 bits: codes m n k.  Prints a line a call: "ok" and figures, or what is wrong.
#include "../paper_2204_03643_amd/csrc/tv_block_plan.hpp"
#include "../paper_2204_03643_amd/csrc/tv_linear4_plan.hpp"
#include <cstdio>

using namespace tvl;

static const char *units_wrong(const Units &u, int64_t m, bool shared, int64_t div)
{
    int64_t next = 0;
    for (int i = 0; i < u.count; ++i) {
        int64_t begin, end;
        range_of(u, i, m, begin, end);
        if (begin != next) return "rows left out, or met twice";
        if (end <= begin || end > m) return "a unit without rows, or beyond them";
        if (shared && u.cuts > 1 && begin / div != (end - 1) / div) return "a unit of two gates";
        if (shared && u.cuts > 1 && i / u.cuts != begin / div) return "a gate's units do not lie together";
        if (shared && u.cuts == 1 && begin % div != 0) return "a unit that starts within a gate";
        next = end;
    }
    return next == m ? nullptr : "rows left out at the end";
}

int main()
{
    long long m, n, shared, div, codes, k;
    while (scanf("%lld %lld %lld %lld", &m, &n, &shared, &div) == 4 && n) {
        const Units u = block_units(m, n, shared != 0, div);
        const char *wrong = units_wrong(u, m, shared != 0, div);
        if (!wrong && (int64_t)u.count * (block_lanes(n) > 64 ? block_lanes(n) : 64) >= (int64_t)1 << 32) wrong = "too many threads";
        tv_block_in in{};
        tv_block_grads g{};
        tv_block_desc d{};
        char there;
        in.x = in.f = in.gate = in.bias = &there;
        g.dweight = g.dbias = g.dscale = g.dgate = g.dnext_weight = g.dnext_bias = &there;
        d.m = m; d.n = n; d.gate_div = shared ? div : 1; d.norm = d.next_norm = TV_NORM_LAYER;
        const BlockBwdPlan p = block_bwd_plan(in, g, d);
        const int64_t each = block_lanes(n) < 64 ? 64 / block_lanes(n) : 1;
        if (!wrong && (p.parts * each < p.units.count || (p.parts - 1) * each >= p.units.count) && p.units.count) wrong = "units without a workgroup";
        if (!wrong && p.bytes < (size_t)(5 * (int64_t)p.parts + (p.want >> kVectors & 1 ? p.units.count : 0)) * n * 4) wrong = "a workspace that is too small";
        if (!wrong && block_lanes(n) > kMostSumLanes && p.two_passes != (p.slots > kMostSlots || n > 8192)) wrong = "the wrong passes";
        if (!wrong && u.cuts > 1 && m / div + kVectors > 65535) wrong = "too many sums to join in a launch";
        if (wrong) printf("%s\n", wrong);
        else printf("ok %d %d %d\n", u.count, u.rows, u.cuts);
    }
    while (scanf("%lld %lld %lld %lld", &codes, &m, &n, &k) == 4) {
        tv_linear_desc d{};
        d.m = m; d.n = n; d.k = k;
        const Plan4 p = plan4(d, codes != 0);
        const int64_t groups = groups_of(k), per = p.c.k_per / 32;
        const Tile side = p.c.kind == kTile256x4 ? Tile{256, 256} : p.c.kind == kTile128x4 ? Tile{128, 128} : Tile{64, 128};
        const int64_t workgroups = p.c.kind == kFew4 ? tiles(n, 16) : tiles(m, side.m) * tiles(n, side.n);
        const int64_t threads = workgroups * p.c.splits * (p.c.kind == kFew4 || p.c.kind == kTile256x4 ? 512 : 256);
        const char *wrong = nullptr;
        if (threads >= (int64_t)1 << 32) wrong = "too many threads";
        if (p.c.kind == kFew4 && (m > kFewRows4 || p.c.splits != 1 || (p.c.own && (codes || m > 16)))) wrong = "a stream of too many rows, or split";
        if (p.c.kind != kFew4 && (per % 2 != 0 || (p.c.splits - 1) * per >= groups || p.c.splits * per < groups)) wrong = "splits that do not cover the contraction";
        if (p.c.kind != kFew4 && (int64_t)(side.m > side.n ? side.m : side.n) * groups * 64 >= (int64_t)1 << 32) wrong = "a tile that spans 2^32 bytes";
        const size_t x = codes || p.c.own ? 0 : (size_t)(m * groups * 64 + scale_rows(m) * groups * 4);
        const size_t sums = p.c.splits > 1 ? (size_t)p.c.splits * m * up(n, 8) * 4 : 0;
        if (p.bytes < x + sums || p.split % 16 || p.exps % 16) wrong = "a workspace that is too small";
        if (wrong) printf("%s\n", wrong);
        else printf("ok %d %d %d\n", (int)p.c.kind, (int)p.c.own, p.c.splits);
    }
    return 0;
}
