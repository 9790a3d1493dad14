// C-ABI entry points of residual borders and dropout: argument validation and launches.
#include "../../include/tvprox.h"
#include "tv_block.hpp"
#include "tv_block_plan.hpp"

namespace {

using namespace tvl;

int launched() { return hipGetLastError() == hipSuccess ? TV_OK : TV_ERR_HIP; }

constexpr int64_t kMostGroups = 8192;        // workgroups of a launch: 32 a compute unit; they take further rows in turn

int check_drop(const tv_drop &d)
{
    if (d.drop > 65536u) return TV_ERR_UNSUPPORTED;
    return aligned(d.seed_at, 8) ? TV_OK : TV_ERR_STRIDE;
}

Drop drop_of(const tv_drop &d)
{
    return {d.seed, d.offset, d.seed_at, d.drop, d.drop < 65536u ? 65536.0f / (float)(65536u - d.drop) : 0.0f};
}

int check_sizes(const tv_block_in &in, const tv_block_desc &d)
{
    if (d.m < 0 || d.n < 1 || d.m >= kMostIndex) return TV_ERR_SHAPE;
    if (in.f && in.gate && (d.gate_div < 1 || d.gate_div >= kMostIndex || d.m % d.gate_div != 0)) return TV_ERR_SHAPE;
    if (d.n > TV_MAX_LENGTH || (d.dtype != TV_F32 && d.dtype != TV_BF16)) return TV_ERR_UNSUPPORTED;
    if (d.next_norm < TV_NORM_NONE || d.next_norm > TV_NORM_LAYER || !(d.eps >= 0.0f)) return TV_ERR_UNSUPPORTED;
    if (d.ldx < d.n || d.ldx >= kMostStride) return TV_ERR_STRIDE;
    if (in.f) {
        if (d.norm < TV_NORM_NONE || d.norm > TV_NORM_LAYER || d.gate_act < TV_GATE_PLAIN || d.gate_act > TV_GATE_SILU) return TV_ERR_UNSUPPORTED;
        if (d.ldf < d.n || d.ldf >= kMostStride) return TV_ERR_STRIDE;
        if (in.gate && (d.ldg < d.n || d.ldg >= kMostStride)) return TV_ERR_STRIDE;
        if (d.remake_y && (d.remake_y != 1 || d.dtype != TV_BF16)) return TV_ERR_UNSUPPORTED;
        return check_drop(d.drop);
    }
    return TV_OK;
}

bool all_aligned(std::initializer_list<const void *> ps, size_t to)
{
    for (const void *p : ps)
        if (!aligned(p, to)) return false;
    return true;
}

bool in_aligned(const tv_block_in &in, size_t to)
{
    return all_aligned({in.x, in.next_weight, in.next_bias}, to) &&
           (!in.f || all_aligned({in.f, in.weight, in.bias, in.gate, in.scale}, to));
}

Block block_of(const tv_block_in &in, const tv_block_desc &d)
{
    Block a{};
    a.x = in.x; a.nw = in.next_weight; a.nb = in.next_bias;
    a.m = d.m; a.ldx = d.ldx;
    a.n = (int32_t)d.n; a.next = d.next_norm;
    a.eps = d.eps; a.inv_n = 1.0f / (float)d.n;
    a.gate_div = 1;
    if (in.f) {
        a.f = in.f; a.gate = in.gate; a.scale = in.scale;
        a.w = d.norm ? in.weight : nullptr; a.b = d.norm ? in.bias : nullptr;
        a.ldf = d.ldf;
        if (in.gate) a.ldg = d.ldg, a.gate_div = (int32_t)d.gate_div;
        a.norm = d.norm; a.act = d.gate_act;
        a.again = d.remake_y != 0;
        a.drop = drop_of(d.drop);
    }
    return a;
}

template <class T, int LANES>
int launch_fwd(const Block &a, void *y, void *h, float *stats, hipStream_t stream)
{
    constexpr int kThreads = LANES > 64 ? LANES : 256;
    const int64_t groups = tiles(a.m, kThreads / LANES);
    const dim3 grid((uint32_t)(groups < kMostGroups ? groups : kMostGroups)), block(kThreads);
    const bool tail = a.n % 8 != 0;
    if (a.f && a.next) hipLaunchKernelGGL((tail ? block_fwd_kernel<T, LANES, true, true, true> : block_fwd_kernel<T, LANES, true, true, false>), grid, block, 0, stream, a, (T *)y, (T *)h, (float4 *)stats);
    else if (a.f) hipLaunchKernelGGL((tail ? block_fwd_kernel<T, LANES, true, false, true> : block_fwd_kernel<T, LANES, true, false, false>), grid, block, 0, stream, a, (T *)y, (T *)h, (float4 *)stats);
    else hipLaunchKernelGGL((tail ? block_fwd_kernel<T, LANES, false, true, true> : block_fwd_kernel<T, LANES, false, true, false>), grid, block, 0, stream, a, (T *)y, (T *)h, (float4 *)stats);
    return launched();
}

template <class T>
int launch_fwd_long(const Block &a, void *y, void *h, float *stats, hipStream_t stream)
{
    const dim3 grid((uint32_t)(a.m < kMostGroups ? a.m : kMostGroups)), block(1024);
    if (a.f && a.next) hipLaunchKernelGGL((block_fwd_long_kernel<T, 1024, 2, true, true>), grid, block, 0, stream, a, (T *)y, (T *)h, (float4 *)stats);
    else if (a.f) hipLaunchKernelGGL((block_fwd_long_kernel<T, 1024, 2, true, false>), grid, block, 0, stream, a, (T *)y, (T *)h, (float4 *)stats);
    else hipLaunchKernelGGL((block_fwd_long_kernel<T, 1024, 2, false, true>), grid, block, 0, stream, a, (T *)y, (T *)h, (float4 *)stats);
    return launched();
}

template <class T>
int block_fwd(const Block &a, void *y, void *h, float *stats, hipStream_t stream)
{
    switch (block_lanes(a.n)) {
    case 8: return launch_fwd<T, 8>(a, y, h, stats, stream);
    case 16: return launch_fwd<T, 16>(a, y, h, stats, stream);
    case 32: return launch_fwd<T, 32>(a, y, h, stats, stream);
    case 64: return launch_fwd<T, 64>(a, y, h, stats, stream);
    case 128: return launch_fwd<T, 128>(a, y, h, stats, stream);
    case 256: return launch_fwd<T, 256>(a, y, h, stats, stream);
    case 512: return launch_fwd<T, 512>(a, y, h, stats, stream);
    default: return a.n <= 8192 ? launch_fwd<T, 1024>(a, y, h, stats, stream) : launch_fwd_long<T>(a, y, h, stats, stream);
    }
}

template <class T, int LANES, int SLOTS>
int launch_bwd(const Block &a, const BlockGrads &o, hipStream_t stream)
{
    const dim3 grid((uint32_t)o.parts), block(LANES > 64 ? LANES : 64);
    const bool tail = a.n % 8 != 0;
    if (a.f && a.next) hipLaunchKernelGGL((tail ? block_bwd_kernel<T, LANES, true, true, true, SLOTS> : block_bwd_kernel<T, LANES, true, true, false, SLOTS>), grid, block, 0, stream, a, o);
    else if (a.f) hipLaunchKernelGGL((tail ? block_bwd_kernel<T, LANES, true, false, true, SLOTS> : block_bwd_kernel<T, LANES, true, false, false, SLOTS>), grid, block, 0, stream, a, o);
    else if constexpr (SLOTS <= 2)                   // (two sums are all that a norm alone has)
        hipLaunchKernelGGL((tail ? block_bwd_kernel<T, LANES, false, true, true, SLOTS> : block_bwd_kernel<T, LANES, false, true, false, SLOTS>), grid, block, 0, stream, a, o);
    return launched();
}

template <class T, int V>
int launch_rows(const Block &a, const BlockGrads &o, hipStream_t stream)
{
    const dim3 grid((uint32_t)(a.m < kMostGroups ? a.m : kMostGroups)), block(1024);
    if (a.f && a.next) hipLaunchKernelGGL((block_rows_kernel<T, 1024, V, true, true>), grid, block, 0, stream, a, o);
    else if (a.f) hipLaunchKernelGGL((block_rows_kernel<T, 1024, V, true, false>), grid, block, 0, stream, a, o);
    else hipLaunchKernelGGL((block_rows_kernel<T, 1024, V, false, true>), grid, block, 0, stream, a, o);
    return launched();
}

template <class T>
int block_bwd(const Block &a, BlockGrads o, const tv_block_grads &g, const BlockBwdPlan &p, hipStream_t stream)
{
    int st = TV_OK;
    switch (a.m > 0 ? block_lanes(a.n) : 0) {
    case 0: break;
    case 8: st = launch_bwd<T, 8, 0>(a, o, stream); break;
    case 16: st = launch_bwd<T, 16, 0>(a, o, stream); break;
    case 32: st = launch_bwd<T, 32, 0>(a, o, stream); break;
    case 64: st = launch_bwd<T, 64, 0>(a, o, stream); break;
    case 128: st = launch_bwd<T, 128, 0>(a, o, stream); break;
    case 256: st = launch_bwd<T, 256, 0>(a, o, stream); break;
    case 512: st = launch_bwd<T, 512, 0>(a, o, stream); break;
    default: {
        if (!p.two_passes) {
            st = p.slots <= 2 ? launch_bwd<T, 1024, 2>(a, o, stream) : launch_bwd<T, 1024, kMostSlots>(a, o, stream);
            break;
        }
        // rows first; then the sums over them
        st = a.n <= 8192 ? launch_rows<T, 1>(a, o, stream) : launch_rows<T, 2>(a, o, stream);
        if (st != TV_OK || !(p.want || (o.dgate && a.gate_div > 1))) break;
        const dim3 grid((uint32_t)tiles(a.n, 2048), (uint32_t)o.units.count), block(256);
        if (a.f && a.next) hipLaunchKernelGGL((block_sums_kernel<T, true, true>), grid, block, 0, stream, a, o);
        else if (a.f) hipLaunchKernelGGL((block_sums_kernel<T, true, false>), grid, block, 0, stream, a, o);
        else hipLaunchKernelGGL((block_sums_kernel<T, false, true>), grid, block, 0, stream, a, o);
        st = launched();
    }
    }
    if (st != TV_OK || !p.want) return st;
    void *const to[kVectors] = {g.dweight, g.dbias, g.dscale, g.dnext_weight, g.dnext_bias};
    Joins j{};
    const float *from = o.sums;
    for (int k = 0; k < kVectors; ++k)
        if (p.want >> k & 1) {
            j.from[j.vectors] = from;
            j.to[j.vectors++] = to[k];
            from += (int64_t)p.parts * a.n;
        }
    int64_t sums = j.vectors;
    if (p.want >> kVectors & 1) {
        j.gate_from = from;
        j.gate_to = g.dgate;
        sums += a.m / a.gate_div;
    }
    j.parts = p.parts; j.cuts = p.units.cuts; j.n = a.n;
    if (sums == 0) return TV_OK;
    hipLaunchKernelGGL((block_join_kernel<T>), dim3((uint32_t)tiles(a.n, 32), (uint32_t)sums), dim3(1024), 0, stream, j);
    return launched();
}

}  // namespace

extern "C" {

int tv_drop_apply(const void *x, void *y, int64_t rows, int64_t n, int64_t ldx, int dtype, tv_drop drop, hipStream_t stream)
{
    if (rows < 0 || n < 1 || rows >= kMostIndex || n >= kMostIndex) return TV_ERR_SHAPE;
    if (dtype != TV_F32 && dtype != TV_BF16) return TV_ERR_UNSUPPORTED;
    if (ldx < n || ldx >= kMostStride) return TV_ERR_STRIDE;
    const int st = check_drop(drop);
    if (st != TV_OK || rows == 0) return st;
    if (!x || !y) return TV_ERR_NULL;
    if (!all_aligned({x, y}, elem_bytes(dtype))) return TV_ERR_STRIDE;
    // as many lanes a row as leave the fewest idle
    const int64_t per = tiles(n, 8);
    int shift = 8;
    for (int s = 7; s >= 3; --s)
        if (up(per, (int64_t)1 << s) < up(per, (int64_t)1 << shift)) shift = s;
    const int64_t groups = tiles(rows, 256 >> shift);
    const dim3 grid((uint32_t)(groups < kMostGroups ? groups : kMostGroups));
    const Drop d = drop_of(drop);
    if (dtype == TV_BF16)
        hipLaunchKernelGGL((dropout_kernel<bf16>), grid, dim3(256), 0, stream, (const bf16 *)x, (bf16 *)y, rows, (int)n, ldx, shift, d);
    else
        hipLaunchKernelGGL((dropout_kernel<float>), grid, dim3(256), 0, stream, (const float *)x, (float *)y, rows, (int)n, ldx, shift, d);
    return launched();
}

int tv_block_fwd(tv_block_in in, void *y, void *h, float *stats, tv_block_desc d, hipStream_t stream)
{
    const int st = check_sizes(in, d);
    if (st != TV_OK) return st;
    if ((!in.f && y) || (h && d.next_norm == TV_NORM_NONE)) return TV_ERR_UNSUPPORTED;
    if (d.m == 0) return TV_OK;
    if (!in.x || (!h && d.next_norm != TV_NORM_NONE) || (!y && !h)) return TV_ERR_NULL;
    const size_t size = elem_bytes(d.dtype);
    if (!in_aligned(in, size) || !all_aligned({y, h}, size) || !aligned(stats, 16)) return TV_ERR_STRIDE;
    const Block a = block_of(in, d);
    return d.dtype == TV_BF16 ? block_fwd<bf16>(a, y, h, stats, stream) : block_fwd<float>(a, y, h, stats, stream);
}

size_t tv_block_bwd_workspace_bytes(tv_block_in in, tv_block_grads grads, tv_block_desc d)
{
    return check_sizes(in, d) == TV_OK ? block_bwd_plan(in, grads, d).bytes : 0;
}

int tv_block_bwd(const void *dy, const void *dh, tv_block_in in, const float *stats, tv_block_grads g, tv_block_desc d,
                 void *ws, size_t ws_bytes, hipStream_t stream)
{
    const int st = check_sizes(in, d);
    if (st != TV_OK) return st;
    if (dh && d.next_norm == TV_NORM_NONE) return TV_ERR_UNSUPPORTED;
    if (!in.f && (g.df || g.dgate || g.dweight || g.dbias || g.dscale)) return TV_ERR_UNSUPPORTED;
    if (in.f && d.norm == TV_NORM_NONE && (g.dweight || g.dbias)) return TV_ERR_UNSUPPORTED;
    if ((g.dgate && !in.gate) || (d.next_norm == TV_NORM_NONE && (g.dnext_weight || g.dnext_bias))) return TV_ERR_UNSUPPORTED;
    const bool normed = (in.f && d.norm != TV_NORM_NONE) || (dh && d.next_norm != TV_NORM_NONE);
    if (d.m > 0 && ((!dy && !dh) || (dh && !in.x) || (normed && !stats))) return TV_ERR_NULL;
    const size_t size = elem_bytes(d.dtype);
    if (!in_aligned(in, size) || !all_aligned({dy, dh, g.dx, g.df, g.dgate, g.dweight, g.dbias, g.dscale, g.dnext_weight, g.dnext_bias}, size) ||
        !aligned(stats, 16)) return TV_ERR_STRIDE;
    const BlockBwdPlan p = block_bwd_plan(in, g, d);
    if (p.bytes && (!ws || !aligned(ws, 16) || ws_bytes < p.bytes)) return TV_ERR_WORKSPACE;
    const Block a = block_of(in, d);
    BlockGrads o{};
    o.dy = dy; o.dh = dh; o.stats = (const float4 *)stats;
    o.dx = g.dx; o.df = g.df; o.dgate = g.dgate;
    o.sums = (float *)ws;
    o.row_sums = p.bytes > p.row_sums ? (float2 *)((char *)ws + p.row_sums) : nullptr;
    o.want = p.want;
    for (int k = 0; k < kSums; ++k) o.slot[k] = p.slot[k];
    o.parts = p.parts;
    o.units = p.units;
    return d.dtype == TV_BF16 ? block_bwd<bf16>(a, o, g, p, stream) : block_bwd<float>(a, o, g, p, stream);
}

}  // extern "C"
