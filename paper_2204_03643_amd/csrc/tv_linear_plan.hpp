// Which kernels a channel product takes, how its contraction is split and how its workspace is laid out.  Host code alone:
// it needs no GPU compiler.
#pragma once
#include "../../include/tvprox.h"
#include <initializer_list>

namespace tvl {

constexpr int64_t kMostIndex = ((int64_t)1 << 31) - 1024;      // sizes stay below: a step past the end fits 32 bits too
constexpr int64_t kMostStride = (int64_t)1 << 31;              // strides stay below
constexpr int64_t kMostTiles = TV_LINEAR_MAX_TILES;            // so that every launch has fewer than 2^32 threads

inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t tiles(int64_t v, int64_t of) { return (v + of - 1) / of; }
inline size_t elem_bytes(int dtype) { return dtype == TV_BF16 ? 2 : 4; }
inline bool aligned(const void *p, size_t to) { return (uintptr_t)p % to == 0; }

// ---- products
// One operand: `rows` rows of `cols` elements, ld apart.
struct Operand {
    const void *p;
    int64_t ld, rows, cols;
};

// Rows on 16-byte boundaries, whole 16-byte pieces, and offsets within a tile of 256 rows that 32 bits hold.  (Rows that the
// library lays out itself are on such boundaries whatever their length: offsets_fit() says which tiles reach them.)
inline bool direct(const Operand &o)
{
    return aligned(o.p, 16) && o.ld % 8 == 0 && o.cols % 8 == 0 && o.ld <= ((int64_t)1 << 22);
}

constexpr int64_t kFewRows = 64;

// Which kernel a product takes and how its contraction is split.
enum Kind { kFew, kTile256, kTile128, kTile128Deep, kTile64, kSplit256, kSplit128, kSplit64 };
struct Choice {
    Kind kind;
    int splits, k_per;
    double us;           // what the model says
};

struct Tile { int m, n; };
inline Tile tile_of_kind(Kind k)
{
    if (k == kTile256 || k == kSplit256) return {256, 256};
    if (k == kTile64 || k == kSplit64) return {64, 128};
    return {128, 128};
}

// `s` splits of a contraction of K, each a multiple of `unit`
inline Choice cut(Kind kind, int64_t s, int64_t K, int64_t unit)
{
    if (s < 1) s = 1;
    const int64_t per = up(K > 0 ? tiles(K, s) : 1, unit);
    return {kind, (int)(K > 0 ? tiles(K, per) : 1), (int)per, 0.0};
}

// Sizes, type and alignment alone decide.  Few rows stream the weight, where that is faster than tiles.  bf16 operands that
// go straight to LDS: up to 32 rows (2048 -> 8192, streamed and through tiles: 32 rows 11.6 and 12.8 us, 48 rows 14.7 and
// 13.8); f32 ones up to 16 (16 rows 22.7 and 23.2 us, 32 rows 28.4 and 23.8).  More rows, and rows on other boundaries, cost
// so much a turn of the waves that only short streams pay: turns one after the other, times the 2, 3 or 6 that one costs
// with up to 16, 32 or 64 rows, up to 36 in f32 (1024 -> 1024: 32 rows, 24, 9.1 and 12.2 us; 64 rows, 48,
// 14.1 and 12.8) and 12 in bf16 (1001 -> 777, 32 rows, 12: 9.0 and 10.8 us; 2047 -> 513, 16 rows, 16: 15.1 and 11.3).
//
// Otherwise the cheapest by a model of the time in microseconds, fitted to sweeps of tiles and splits over outputs of
// 128 x 512 to 8192 x 8192 and contractions of 256 to 16384 (what it takes there is 0.1 to 0.8 % slower than the best of the sweep, 11 %
// at most): a launch; rounds of workgroups over 256 compute units, in each a start and an end and so much a step of 64,
// more where two workgroups share a unit or, at lower clocks, where more than half of the units are busy; for split
// contractions the second launch and the sums' trip through memory.
struct Cost {
    Kind kind;
    int64_t slots;               // workgroups at a time
    double round, step, more;
};

inline double rounds_us(const Cost &c, int64_t workgroups, int64_t steps)
{
    const int64_t full = workgroups / c.slots, rest = workgroups % c.slots;
    // (the second half of 256 workgroups does not spread evenly where units take two)
    const double half = rest > 128 ? rest / 128.0 - 1.0 : 0.0, load = c.slots == 256 ? half : rest > 256 ? 1.0 : 0.5 * half;
    double us = (double)full * (c.round + (c.step + c.more) * (double)steps);
    if (rest) us += c.round + (c.step + c.more * load) * (double)steps;
    return us;
}

// The strides of a product's operands, and which of them have the output index contiguous.
struct Layout {
    int64_t lda, ldb;
    bool at, bt;
};

// The kernels that load straight to LDS keep 32-bit offsets from a tile's origin: to the tile's last row and 64 contraction
// indices of it, or to the last contraction index of a step and the tile's columns there.
inline bool offsets_fit(Kind kind, const Layout &l, int64_t M, int64_t N)
{
    const Tile side = tile_of_kind(kind);
    const int64_t a = l.at ? 63 * l.lda + side.m : ((M < side.m ? M : side.m) - 1) * l.lda + 64;
    const int64_t b = l.bt ? 63 * l.ldb + side.n : ((N < side.n ? N : side.n) - 1) * l.ldb + 64;
    return a * 2 < (int64_t)1 << 32 && b * 2 < (int64_t)1 << 32;
}

inline Choice choose_tiles(int dtype, bool direct, const Layout &l, int64_t M, int64_t N, int64_t K)
{
    constexpr Cost direct16[] = {{kTile64, 256, 1.0, 0.25, 0.08}, {kTile128Deep, 256, 1.8, 0.38, 0.13}, {kTile128, 512, 1.5, 0.42, 0.52}, {kTile256, 256, 4.2, 1.14, 0.49}};
    constexpr Cost any16[] = {{kSplit64, 512, 3.2, 0.45, 0.44}};
    constexpr Cost any32[] = {{kSplit64, 256, 4.2, 1.26, 0.35}, {kSplit128, 256, 3.6, 1.97, 0.80}, {kSplit256, 256, 7.4, 6.6, 2.5}};
    const Cost *costs = dtype != TV_BF16 ? any32 : direct ? direct16 : any16;
    const int kinds = dtype != TV_BF16 ? 3 : direct ? 4 : 1;
    Choice best = cut(costs[0].kind, 1, K, 64);
    best.us = 1e30;
    for (int i = 0; i < kinds; ++i) {
        const Cost &c = costs[i];
        if (costs == direct16 && !offsets_fit(c.kind, l, M, N)) continue;
        const Tile side = tile_of_kind(c.kind);
        const int64_t t = tiles(M, side.m) * tiles(N, side.n);
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
            if (s > 1 && (K < 128 * s || t * s > 1024)) break;
            Choice x = cut(c.kind, s, K, 64);
            x.us = 3.0 + rounds_us(c, t * x.splits, tiles(x.k_per < K ? x.k_per : K, 64));
            if (x.splits > 1) x.us += 2.6 + 0.18 * x.splits + (double)M * (double)N * x.splits * 8 / 7e6;
            if (x.us < best.us) best = x;
        }
    }
    if (best.us == 1e30) return choose_tiles(dtype, false, l, M, N, K);      // (rows too long for all of them: 64-bit addresses)
    return best;
}

inline Choice choose(int dtype, bool direct, const Layout &l, int64_t M, int64_t N, int64_t K)
{
    if (!l.at && !l.bt && M >= 1 && M <= kFewRows) {
        const int64_t turn = 8 * 64 / (int64_t)elem_bytes(dtype);            // a turn of all eight waves
        const int64_t t = tiles(N, 32), s = t >= 256 ? 1 : 256 / t;
        const Choice x = cut(kFew, s < K / (8 * turn) ? s : K / (8 * turn), K, turn);
        const int64_t turns = tiles(t * x.splits, 256) * tiles(x.k_per < K ? x.k_per : K, turn);
        if ((direct && M <= (dtype == TV_BF16 ? 32 : 16)) || turns * (M <= 16 ? 2 : M <= 32 ? 3 : 6) <= (dtype == TV_BF16 ? 12 : 36)) return x;
    }
    return choose_tiles(dtype, direct, l, M, N, K);
}

// bf16 operands that cannot go straight to LDS are copied to rows that can, where the faster kernel pays for it
// (8192 x 2047 -> 8191: 505 us without, 250 with): a launch and the bytes there and back each.
struct Plan {
    Choice c;
    bool copy_a, copy_b;
};
inline double copy_us(int64_t rows, int64_t cols) { return 4.0 + (double)rows * (double)cols * 4 / 4e6; }

inline Plan plan(int dtype, bool direct_a, bool direct_b, const Layout &l, int64_t M, int64_t N, int64_t K)
{
    Plan p{choose(dtype, direct_a && direct_b, l, M, N, K), false, false};
    if (dtype != TV_BF16 || (direct_a && direct_b) || p.c.kind == kFew || M < 1 || K < 1) return p;
    const Layout copied{direct_a ? l.lda : up(l.at ? M : K, 8), direct_b ? l.ldb : up(l.bt ? N : K, 8), l.at, l.bt};
    Choice c = choose_tiles(dtype, true, copied, M, N, K);
    c.us += (direct_a ? 0.0 : copy_us(M, K)) + (direct_b ? 0.0 : copy_us(N, K));
    return c.us < p.c.us ? Plan{c, !direct_a, !direct_b} : p;
}

inline int64_t copy_bytes(int64_t rows, int64_t cols) { return up(rows * up(cols, 8) * 2, 256); }

inline size_t split_bytes(const Choice &c, int64_t M, int64_t N)
{
    return c.splits > 1 ? (size_t)up((int64_t)c.splits * M * up(N, 8) * 4, 256) : 0;
}

inline bool product_fits(int64_t M, int64_t N) { return tiles(M, 128) * tiles(N, 128) <= kMostTiles; }

// ---- the forward call's workspace: copies of x and W, split sums
struct FwdPlan {
    Plan product;
    size_t w, split, bytes;
};

inline FwdPlan fwd_plan(const tv_linear_desc &d, bool direct_x, bool direct_w)
{
    FwdPlan p{};
    p.product = plan(d.dtype, direct_x, direct_w, {d.ldx, d.ldw, false, false}, d.m, d.n, d.k);
    p.w = p.product.copy_a ? copy_bytes(d.m, d.k) : 0;
    p.split = p.w + (p.product.copy_b ? copy_bytes(d.n, d.k) : 0);
    p.bytes = p.split + split_bytes(p.product.c, d.m, d.n);
    return p;
}

// ---- the backward call's workspace: dz (or a copy of g), x out of its checkpoint or a copy of it, a copy of W, the column
// sums of groups of rows, split sums
struct BwdPlan {
    Plan dx, dw;
    size_t x, w, sums, split, bytes;
    int64_t ldz, ldx;
    int rows_per, groups;
    bool own_dz, own_x;
};

struct Wanted { bool dx, dw, db; };

inline BwdPlan bwd_plan(const tv_linear_desc &d, bool x8, bool direct_g, bool direct_x, bool direct_w, Wanted want)
{
    BwdPlan p{};
    const int64_t size = (int64_t)elem_bytes(d.dtype);
    const bool smooth = d.act != TV_ACT_NONE;
    p.ldz = up(d.n, 8);
    p.ldx = up(d.k, 8);
    // dz is written, and codes are restored, into rows that go straight to LDS
    const int64_t ldz = smooth ? p.ldz : d.ldy, ldx = x8 ? p.ldx : d.ldx;
    p.dx = plan(d.dtype, smooth || direct_g, direct_w, {ldz, d.ldw, false, true}, d.m, d.k, d.n);
    p.dw = plan(d.dtype, smooth || direct_g, x8 || direct_x, {ldz, ldx, true, true}, d.n, d.k, d.m);
    p.own_dz = (want.dx && (smooth || p.dx.copy_a)) || (want.dw && (smooth || p.dw.copy_a));
    p.own_x = want.dw && (x8 || p.dw.copy_b);
    size_t at = p.own_dz ? up(d.m * p.ldz * size, 256) : 0;
    p.x = at;
    if (p.own_x) at += copy_bytes(d.m, d.k);
    p.w = at;
    if (want.dx && p.dx.copy_b) at += copy_bytes(d.n, d.k);
    // about 1024 workgroups of 256 columns each, of sixteen rows at least; up to 64 rows are one group, one launch
    const int64_t share = 1024 / tiles(d.n, 256) + 1;
    p.rows_per = (int)(d.m > 64 ? up(tiles(d.m, share < 256 ? share : 256), 16) : 64);
    p.groups = (int)tiles(d.m, p.rows_per);
    p.sums = at;
    if (want.db) at += up((int64_t)p.groups * d.n * 4, 256);
    p.split = at;
    const size_t s1 = want.dx ? split_bytes(p.dx.c, d.m, d.k) : 0, s2 = want.dw ? split_bytes(p.dw.c, d.n, d.k) : 0;
    p.bytes = at + (s1 > s2 ? s1 : s2);
    return p;
}

}  // namespace tvl
