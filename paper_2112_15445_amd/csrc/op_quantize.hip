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

// One workgroup per block of R x 128 values.
template <int XT, int R> __global__ __launch_bounds__(256) void quantize_kernel(QuantArgs a, int64_t blocks)
{
    __shared__ float red[4];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t item = R == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
    if (item >= blocks) return;
    const int b = (int)(item % a.KB);
    const int64_t m0 = item / a.KB * R;
    const int rows = R == 1 ? 1 : (int)min((int64_t)R, a.M - m0);
    const int c0 = b * kQBlock + lane * 2;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x);
    float amax = kAmaxFloor;
    for (int r = R == 1 ? 0 : wave; r < rows; r += 4)
        for (int i = 0; i < 2; ++i)
            if (c0 + i < a.K) amax = fmaxf(amax, fabsf((float)x[(m0 + r) * a.x_row + c0 + i]));
    for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
    if constexpr (R > 1) {
        if (lane == 0) red[wave] = amax;
        __syncthreads();
        amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    }
    const float up = kCodeMax / amax;
    for (int r = R == 1 ? 0 : wave; r < rows; r += 4)
        for (int i = 0; i < 2; ++i)
            if (c0 + i < ((a.K + 15) & ~15)) {
                const float v = c0 + i < a.K ? (float)x[(m0 + r) * a.x_row + c0 + i] : 0.0f;
                a.q[(m0 + r) * a.q_row + c0 + i] = code1(v * up);
            }
    if (lane == 0 && (R == 1 || wave == 0)) a.scale[item / a.KB * a.s_row + b] = amax / kCodeMax;
}

template <int XT> sc_status_t launch_quantize(const QuantArgs& a, int rows, hipStream_t stream)
{
    const int64_t blocks = ceil_div(a.M, rows) * a.KB;
    if (rows == 1) quantize_kernel<XT, 1><<<dim3((unsigned)ceil_div(blocks, 4)), 256, 0, stream>>>(a, blocks);
    else quantize_kernel<XT, 128><<<dim3((unsigned)blocks), 256, 0, stream>>>(a, blocks);
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
    if (ceil_div(d->M, d->rows) * ceil_div(d->K, kQBlock) >= (int64_t)1 << 31) return SC_ERR_RANGE;
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
