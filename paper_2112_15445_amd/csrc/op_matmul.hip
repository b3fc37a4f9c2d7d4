// Products in blocks (sparse_conv_matmul_blocks) and grouped by expert (sparse_conv_matmul_grouped).
#include "op_matmul_kernel.h"

#include <algorithm>
#include <cmath>

namespace sc {
namespace {

template <int AT, int YT, bool GROUPED, int BT, int BN, int WT, int WN, int ST, int KS = 1> sc_status_t launch_tile(const MatmulArgs& p, hipStream_t stream)
{
    const int64_t tiles = (ceil_div(p.M, BT) + (GROUPED ? std::min(p.E, p.M) : 0)) * ceil_div(p.N, BN);
    if (tiles * WT * WN * KS * 64 >= (int64_t)1 << 32) return SC_ERR_RANGE;
    matmul_tile_kernel<AT, YT, GROUPED, BT, BN, WT, WN, ST, KS><<<dim3((unsigned)tiles), WT * WN * KS * 64, 0, stream>>>(p);
    return launched();
}

// Waves that share the summed dimension: as many as have kAtOnce slabs each, up to 8.
template <int AT, int YT, bool GROUPED> sc_status_t launch_rows(const MatmulArgs& p, hipStream_t stream)
{
    const int64_t tiles = (ceil_div(p.M, 16) + (GROUPED ? std::min(p.E, p.M) : 0)) * ceil_div(p.N, 16);
    const int waves = (int)std::min<int64_t>(8, ceil_div(ceil_div(p.kbytes, kSlab), kAtOnce));
    if (tiles * waves * 64 >= (int64_t)1 << 32) return SC_ERR_RANGE;
    matmul_rows_kernel<AT, YT, GROUPED><<<dim3((unsigned)tiles), waves * 64, waves * 1024, stream>>>(p);
    return launched();
}

// Which form.  Few rows: where its workgroups (16 x 16 of y) are at most two a compute unit (1 x 4096 x 4096: 7 us against 11 on
// 64 x 64 tiles; 32 rows of that, four a unit: 11.6 against 11.6), and for products of up to 16 rows.  Else the tile whose estimate is
// smallest: a fixed part, and per round of workgroups that are resident together a start and a time per slab, which is shorter in a last
// round that leaves half of the places empty.  The constants, in microseconds, are fitted to 311 products of 1 to 16384 rows, 4 to 64
// groups, 200 to 3200 columns and 256 to 4096 summed values in every pair of types; there the choice costs 2.1 % more than the fastest form
// each time, without the split 64 tile 3.2 %; on 199 of them, timed again, 1.7 %, without the widest 2.3 %, the deep one 2.7 %, the 64 or the 128
// tile 6 %.  Groups: half a tile more each, and one each at least where they have rows (2.0 % on 140 of them, 2.5 % without the latter).
struct TileTime { sc_form_t form; int size, places; double start, slab, slab_half_empty; };
constexpr TileTime kTiles[] = {{SC_FORM_TILE_64, 64, 512, 1.5, 0.41, 0.20},
                               {SC_FORM_TILE_64_SPLIT, 64, 256, 2.3, 0.24, 0.16},
                               {SC_FORM_TILE_128, 128, 512, 3.6, 0.88, 0.67},
                               {SC_FORM_TILE_128_DEEP, 128, 256, 2.2, 0.62, 0.50},
                               {SC_FORM_TILE_256, 256, 256, 6.2, 1.38, 1.25}};

sc_form_t pick_form(const MatmulArgs& p, bool grouped, bool widest)
{
    const int64_t columns16 = ceil_div(p.N, 16), slabs = ceil_div(p.kbytes, kSlab);
    if (grouped ? (ceil_div(p.M, 16) + std::min(p.E, p.M)) * columns16 <= 512 : p.M <= 16 || ceil_div(p.M, 16) * columns16 <= 512) return SC_FORM_ROWS;
    sc_form_t best = SC_FORM_ROWS;
    double least = 0.0;
    for (const TileTime& t : kTiles) {
        if (t.form == SC_FORM_TILE_256 && !widest) continue;
        const double even = (double)ceil_div(p.M, t.size), rows = grouped ? std::max(even + 0.5 * p.E, (double)std::min(p.E, p.M)) : even;
        const double tiles = std::ceil(rows) * (double)ceil_div(p.N, t.size);
        const double full = std::floor(tiles / t.places), rest = tiles - full * t.places;
        const double last = rest == 0.0 ? 0.0 : rest <= 0.5 * t.places ? t.slab_half_empty : t.slab;
        const double time = std::max(7.2, 3.0 + slabs * (full * t.slab + last) + (full + (rest > 0.0)) * t.start);
        if (best == SC_FORM_ROWS || time < least) best = t.form, least = time;
    }
    return best;
}

// (32-bit results of codes keep both operands widened in registers: the widest tile has none left)
constexpr bool has_widest(int a_type, int y_type) { return a_type != SC_ELEM_E4M3 || y_type != SC_ELEM_F32; }

template <int AT, int YT, bool GROUPED> sc_status_t launch(const MatmulArgs& p, hipStream_t stream)
{
    constexpr bool WIDEST = has_widest(AT, YT);
    switch (pick_form(p, GROUPED, WIDEST)) {
        case SC_FORM_ROWS: return launch_rows<AT, YT, GROUPED>(p, stream);
        case SC_FORM_TILE_64: return launch_tile<AT, YT, GROUPED, 64, 64, 2, 2, 4>(p, stream);
        case SC_FORM_TILE_64_SPLIT: return launch_tile<AT, YT, GROUPED, 64, 64, 2, 2, 3, 2>(p, stream);
        // (eight waves where their registers leave room for a second workgroup: 3 % less than four over 68 products; 7 % more in 32-bit
        // results of codes)
        case SC_FORM_TILE_128: return launch_tile<AT, YT, GROUPED, 128, 128, WIDEST ? 4 : 2, 2, 2>(p, stream);
        case SC_FORM_TILE_128_DEEP: return launch_tile<AT, YT, GROUPED, 128, 128, 4, 2, 4>(p, stream);
        default: break;
    }
    if constexpr (WIDEST) return launch_tile<AT, YT, GROUPED, 256, 256, 4, 2, 2>(p, stream);
    else return SC_ERR_UNSUPPORTED;
}

constexpr int64_t kMaxRowBytes = (int64_t)1 << 22;     // (256 rows of a tile are addressed with 32 bits)
constexpr int kMaxRows = 1 << 30;
constexpr int64_t kMaxExpert = (int64_t)1 << 48;       // (of elements: 4096 experts are addressed with 64 bits)

sc_status_t check_blocks(const sc_matmul_blocks_t* d)
{
    if (!d) return SC_ERR_NULL;
    const int64_t KB = ceil_div(d->K, kQBlock);
    if (d->M < 0 || d->N <= 0 || d->K <= 0 || d->a_row < d->K || d->b_row < d->K || d->y_row < d->N || d->a_scale_row < KB || d->b_scale_row < KB)
        return SC_ERR_SHAPE;
    if (!is_wide(d->y_type) || d->act < SC_ACT_NONE || d->act > SC_ACT_SILU || d->a_row % 16 || d->b_row % 16) return SC_ERR_UNSUPPORTED;
    if (d->M > kMaxRows || d->a_row >= kMaxRowBytes || d->b_row >= kMaxRowBytes) return SC_ERR_RANGE;
    return SC_OK;
}

sc_status_t check_grouped(const sc_matmul_grouped_t* d)
{
    if (!d) return SC_ERR_NULL;
    const bool codes = d->a_type == SC_ELEM_E4M3;
    if (d->M < 0 || d->N <= 0 || d->K <= 0 || d->E <= 0 || d->E > 4096 || d->a_rows < 0 || d->a_row < d->K || d->b_row < d->K || d->y_row < d->N) return SC_ERR_SHAPE;
    if (d->a_type != SC_ELEM_F16 && d->a_type != SC_ELEM_BF16 && !codes) return SC_ERR_UNSUPPORTED;
    if (!is_wide(d->y_type) || (!codes && d->y_type != d->a_type && d->y_type != SC_ELEM_F32)) return SC_ERR_UNSUPPORTED;
    const int64_t KB = ceil_div(d->K, kQBlock), e = elem_bytes(d->a_type);
    // (distances are compared as they are: multiplied by the element's size or by rows, a large one could pass for a small one)
    if (d->M > kMaxRows || d->a_row >= kMaxRowBytes / e || d->b_row >= kMaxRowBytes / e || (d->E > 1 && d->b_expert >= kMaxExpert)) return SC_ERR_RANGE;
    if (d->b_expert < (d->N - 1) * d->b_row + d->K && d->E > 1) return SC_ERR_SHAPE;
    if (codes && (d->a_scale_row < KB || d->b_scale_row < KB || (d->E > 1 && d->b_scale_expert < ceil_div(d->N, kQBlock) * KB))) return SC_ERR_SHAPE;
    if (d->act < SC_ACT_NONE || d->act > SC_ACT_SILU || d->a_row % (16 / e) || d->b_row % (16 / e) || d->b_expert % (16 / e)) return SC_ERR_UNSUPPORTED;
    return SC_OK;
}

// What the choice of a form goes by.
MatmulArgs sizes(const sc_matmul_blocks_t* d)
{
    MatmulArgs p{};
    p.M = d->M; p.N = d->N; p.E = 1; p.kbytes = d->K;
    return p;
}

MatmulArgs sizes(const sc_matmul_grouped_t* d)
{
    MatmulArgs p{};
    p.M = d->M; p.N = d->N; p.E = d->E; p.kbytes = d->K * elem_bytes(d->a_type);
    return p;
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_matmul_blocks_workspace_size(const sc_matmul_blocks_t* d, size_t* bytes)
{
    if (!bytes) return SC_ERR_NULL;
    const sc_status_t st = check_blocks(d);
    if (st == SC_OK) *bytes = 0;
    return st;
}

extern "C" sc_status_t sparse_conv_matmul_blocks_launch(const sc_matmul_blocks_t* d, sc_launch_t* launch)
{
    if (!launch) return SC_ERR_NULL;
    const sc_status_t st = check_blocks(d);
    if (st != SC_OK) return st;
    *launch = sc_launch_t{};
    if (d->M) launch->form = pick_form(sizes(d), false, has_widest(SC_ELEM_E4M3, d->y_type));
    return SC_OK;
}

extern "C" sc_status_t sparse_conv_matmul_blocks(const sc_matmul_blocks_t* d, const void* a, const float* a_scale, const void* b,
                                                 const float* b_scale, const float* bias, void* y, void* workspace_dev,
                                                 size_t workspace_bytes, void* stream)
{
    (void)workspace_dev; (void)workspace_bytes;
    const sc_status_t st = check_blocks(d);
    if (st != SC_OK) return st;
    if (d->M == 0) return SC_OK;
    if (!a || !a_scale || !b || !b_scale || !y) return SC_ERR_NULL;
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(bias, 4) || !aligned(y, elem_bytes(d->y_type)))
        return SC_ERR_UNSUPPORTED;
    MatmulArgs p = sizes(d);
    p.a = static_cast<const uint8_t*>(a); p.b = static_cast<const uint8_t*>(b); p.as = a_scale; p.bs = b_scale; p.bias = bias; p.y = y;
    p.a_rows = d->M;
    p.a_row = d->a_row; p.b_row = d->b_row; p.y_row = d->y_row; p.as_row = d->a_scale_row; p.bs_row = d->b_scale_row; p.act = d->act;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (d->y_type) {
        case SC_ELEM_F32: return launch<SC_ELEM_E4M3, SC_ELEM_F32, false>(p, s);
        case SC_ELEM_F16: return launch<SC_ELEM_E4M3, SC_ELEM_F16, false>(p, s);
        default: return launch<SC_ELEM_E4M3, SC_ELEM_BF16, false>(p, s);
    }
}

extern "C" sc_status_t sparse_conv_matmul_grouped_workspace_size(const sc_matmul_grouped_t* d, size_t* bytes)
{
    if (!bytes) return SC_ERR_NULL;
    const sc_status_t st = check_grouped(d);
    if (st == SC_OK) *bytes = 0;
    return st;
}

extern "C" sc_status_t sparse_conv_matmul_grouped_launch(const sc_matmul_grouped_t* d, sc_launch_t* launch)
{
    if (!launch) return SC_ERR_NULL;
    const sc_status_t st = check_grouped(d);
    if (st != SC_OK) return st;
    *launch = sc_launch_t{};
    if (d->M) launch->form = pick_form(sizes(d), true, has_widest(d->a_type, d->y_type));
    return SC_OK;
}

extern "C" sc_status_t sparse_conv_matmul_grouped(const sc_matmul_grouped_t* d, const void* a, const float* a_scale,
                                                  const int32_t* index, const int32_t* offsets, const void* b, const float* b_scale,
                                                  const float* bias, void* y, void* workspace_dev, size_t workspace_bytes, void* stream)
{
    (void)workspace_dev; (void)workspace_bytes;
    const sc_status_t st = check_grouped(d);
    if (st != SC_OK) return st;
    if (!index && d->a_rows < d->M) return SC_ERR_SHAPE;
    if (d->M == 0) return SC_OK;
    const bool codes = d->a_type == SC_ELEM_E4M3;
    if ((!a && d->a_rows > 0) || !offsets || !b || !y || (codes && ((!a_scale && d->a_rows > 0) || !b_scale))) return SC_ERR_NULL;
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(bias, 4) || !aligned(index, 4) || !aligned(offsets, 4) ||
        !aligned(y, elem_bytes(d->y_type)))
        return SC_ERR_UNSUPPORTED;
    const int e = elem_bytes(d->a_type);
    MatmulArgs p = sizes(d);
    p.a = static_cast<const uint8_t*>(a); p.b = static_cast<const uint8_t*>(b); p.as = a_scale; p.bs = b_scale; p.bias = bias;
    p.index = index; p.offsets = offsets; p.y = y;
    p.a_rows = d->a_rows;
    p.a_row = d->a_row * e; p.b_row = d->b_row * e; p.b_expert = d->E > 1 ? d->b_expert * e : 0; p.y_row = d->y_row;
    p.as_row = d->a_scale_row; p.bs_row = d->b_scale_row; p.bs_expert = d->b_scale_expert; p.act = d->act;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = d->y_type == SC_ELEM_F32;
    switch (d->a_type) {
        case SC_ELEM_F16: return f32 ? launch<SC_ELEM_F16, SC_ELEM_F32, true>(p, s) : launch<SC_ELEM_F16, SC_ELEM_F16, true>(p, s);
        case SC_ELEM_BF16: return f32 ? launch<SC_ELEM_BF16, SC_ELEM_F32, true>(p, s) : launch<SC_ELEM_BF16, SC_ELEM_BF16, true>(p, s);
        default: break;
    }
    return f32 ? launch<SC_ELEM_E4M3, SC_ELEM_F32, true>(p, s) : d->y_type == SC_ELEM_F16 ? launch<SC_ELEM_E4M3, SC_ELEM_F16, true>(p, s) : launch<SC_ELEM_E4M3, SC_ELEM_BF16, true>(p, s);
}
