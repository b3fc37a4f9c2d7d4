// Quantisation by blocks (sparse_conv_quantize_blocks).
#include "op_common.h"

namespace sc {
namespace {

struct QuantArgs {
    const void* x;
    uint8_t* q;
    float* scale;
    int M, K, KB;
    int64_t x_row, q_row, s_row;
};

// Blocks of one row: 128 values are 16 bytes each of 16 lanes (two-byte types) or 32 (fp32), so that a wave's load is one run of 1 KB;
// the magnitude goes round those lanes by shuffles and the values never leave the registers between the two passes over them.
// Bound by memory: 25088 x 512 f16 (39 MB) takes 8.5 us a call, 4.6 TB/s.  Two blocks a lane are under way at once (four 15 % more, eight 36).
template <int XT> __global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a, uint32_t items)
{
    constexpr int V = kVec<XT>, L = kQBlock / V, U = 2;
    const int part = threadIdx.x % L;
    const uint32_t first = blockIdx.x * (256 / L * U) + threadIdx.x / L;
    v4i raw[U];
    uint32_t row[U];
    int col[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t item = min(first + u * (256 / L), items - 1);
        row[u] = item / (uint32_t)a.KB;
        col[u] = (int)(item - row[u] * (uint32_t)a.KB) * kQBlock + part * V;
        const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + row[u] * a.x_row + col[u];
        raw[u] = col[u] + V <= a.K ? load_raw<XT>(x) : load_raw_part<XT>(x, a.K - col[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[V], amax = kAmaxFloor;
        to_floats<XT>(raw[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) amax = fmaxf(amax, fabsf(f[i]));
        amax = max_block<L>(amax);
        if (first + u * (256 / L) >= items) continue;
        if (col[u] < ((a.K + 15) & ~15)) store_codes<V>(a.q + row[u] * a.q_row + col[u], f, kCodeMax / amax);
        if (part == 0) a.scale[row[u] * a.s_row + col[u] / kQBlock] = amax / kCodeMax;
    }
}

// Blocks of 128 rows: one workgroup each, the whole block in its registers (32 bytes a lane and two-byte type, 64 in fp32).  Bound, where
// there are fewer blocks than compute units, by launch, one burst of loads and one of stores: 2048 x 1100 fp32 (144 blocks, 11 MB) 5.7 us.
template <int XT> __global__ __launch_bounds__(1024) void quantize_tiles_kernel(QuantArgs a)
{
    constexpr int V = kVec<XT>, L = kQBlock / V, R = 1024 / L, U = kQBlock / R;   // lanes of a row, rows at once, rows of a lane
    __shared__ float red[16];
    const int part = threadIdx.x % L;
    const uint32_t tile_row = blockIdx.x / (uint32_t)a.KB, b = blockIdx.x - tile_row * (uint32_t)a.KB;
    const int col = (int)b * kQBlock + part * V;
    const int m0 = (int)tile_row * kQBlock + threadIdx.x / L;
    v4i raw[U];
    float amax = kAmaxFloor;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int m = m0 + u * R;
        const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + m * a.x_row + col;
        raw[u] = v4i{0, 0, 0, 0};
        if (m < a.M) raw[u] = col + V <= a.K ? load_raw<XT>(x) : load_raw_part<XT>(x, a.K - col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[V];
        to_floats<XT>(raw[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) amax = fmaxf(amax, fabsf(f[i]));
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = fmaxf(amax, red[i]);
    const float up = kCodeMax / amax;
    if (col < ((a.K + 15) & ~15))
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int m = m0 + u * R;
            float f[V];
            to_floats<XT>(raw[u], f);
            if (m < a.M) store_codes<V>(a.q + m * a.q_row + col, f, up);
        }
    if (threadIdx.x == 0) a.scale[tile_row * a.s_row + b] = amax / kCodeMax;
}

template <int XT> sc_status_t launch_quantize(const QuantArgs& a, int rows, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.M, rows) * a.KB;
    if (rows == 1) quantize_rows_kernel<XT><<<dim3((unsigned)ceil_div(blocks, 256 / (kQBlock / kVec<XT>) * 2)), 256, 0, stream>>>(a, (uint32_t)blocks);
    else quantize_tiles_kernel<XT><<<dim3((unsigned)blocks), 1024, 0, stream>>>(a);
    return launched();
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_quantize_blocks(const sc_quantize_blocks_t* d, const void* x, void* q, float* scale, void* stream)
{
    if (!d) return SC_ERR_NULL;
    if (d->M < 0 || d->K <= 0 || d->x_row < 0 || d->q_row < d->K || d->scale_row < ceil_div(d->K, kQBlock)) return SC_ERR_SHAPE;
    if ((d->rows != 1 && d->rows != kQBlock) || !is_wide(d->x_type) || d->q_row % 16) return SC_ERR_UNSUPPORTED;
    if (d->K > INT32_MAX - 255) return SC_ERR_RANGE;         // (columns are counted to the end of the last block, in 32 bits)
    if (ceil_div(d->M, d->rows) * ceil_div(d->K, kQBlock) >= (int64_t)1 << (d->rows == 1 ? 27 : 22)) return SC_ERR_RANGE;   // threads of a launch
    if (d->M == 0) return SC_OK;
    if (!x || !q || !scale) return SC_ERR_NULL;
    if (!aligned(x, elem_bytes(d->x_type)) || !aligned(q, 16) || !aligned(scale, 4)) return SC_ERR_UNSUPPORTED;
    QuantArgs a;
    a.x = x; a.q = static_cast<uint8_t*>(q); a.scale = scale;
    a.M = d->M; a.K = d->K; a.KB = (int)ceil_div(d->K, kQBlock);
    a.x_row = d->x_row; a.q_row = d->q_row; a.s_row = d->scale_row;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (d->x_type) {
        case SC_ELEM_F32: return launch_quantize<SC_ELEM_F32>(a, d->rows, s);
        case SC_ELEM_F16: return launch_quantize<SC_ELEM_F16>(a, d->rows, s);
        default: return launch_quantize<SC_ELEM_BF16>(a, d->rows, s);
    }
}
