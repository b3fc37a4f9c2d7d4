// Group norm with an activation, channels last (sparse_conv_group_norm).
#include "op_common.h"

namespace sc {
namespace {

struct NormArgs {
    const void* x;
    const float* gamma;
    const float* beta;
    void* y;
    float* ys;
    float2* stats;
    int S, C, G, Cg, NB;
    float eps;
    int64_t x_sample, x_row, y_sample, y_row, s_row;
};

__device__ __forceinline__ float block_sum(float v, float* red)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[w] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < (int)(blockDim.x >> 6); ++i) s += red[i];
    return s;
}

// One workgroup per (sample, group): mean, then the sum of squared deviations.
template <int XT> __global__ __launch_bounds__(256) void norm_stats_kernel(NormArgs a)
{
    __shared__ float red[4];
    const int n = blockIdx.x / a.G, g = blockIdx.x % a.G;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + g * a.Cg;
    const int64_t cnt = (int64_t)a.S * a.Cg;
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < cnt; i += 256) s += (float)x[i / a.Cg * a.x_row + i % a.Cg];
    const float mean = block_sum(s, red) / (float)cnt;
    float m2 = 0.0f;
    for (int64_t i = threadIdx.x; i < cnt; i += 256) {
        const float d = (float)x[i / a.Cg * a.x_row + i % a.Cg] - mean;
        m2 += d * d;
    }
    m2 = block_sum(m2, red);
    if (threadIdx.x == 0) a.stats[blockIdx.x] = make_float2(mean, 1.0f / sqrtf(m2 / (float)cnt + a.eps));
}

// One wave per (position, 128 channels), two channels a lane.
template <int XT, int YT, int ACT> __global__ __launch_bounds__(256) void norm_apply_kernel(NormArgs a, int64_t items)
{
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (item >= items) return;
    const int b = (int)(item % a.NB);
    const int64_t pos = item / a.NB;
    const int64_t n = pos / a.S, s = pos % a.S;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + s * a.x_row;
    float v[2];
    float amax = kAmaxFloor;
    for (int i = 0; i < 2; ++i) {
        const int c = b * kQBlock + lane * 2 + i;
        v[i] = 0.0f;
        if (c < a.C) {
            const float2 st = a.stats[n * a.G + c / a.Cg];
            float z = ((float)x[c] - st.x) * st.y * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f);
            v[i] = activate<ACT>(z);
        }
        amax = fmaxf(amax, fabsf(v[i]));
    }
    Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + n * a.y_sample + s * a.y_row;
    if constexpr (YT == SC_ELEM_E4M3) {
        for (int o = 32; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
        const float up = kCodeMax / amax;
        for (int i = 0; i < 2; ++i) {
            const int c = b * kQBlock + lane * 2 + i;
            if (c < ((a.C + 15) & ~15)) y[c] = code1(v[i] * up);
        }
        if (lane == 0) a.ys[pos * a.s_row + b] = amax / kCodeMax;
    } else {
        for (int i = 0; i < 2; ++i) {
            const int c = b * kQBlock + lane * 2 + i;
            if (c < a.C) y[c] = (Elem<YT>)v[i];
        }
    }
}

sc_status_t check_norm(const sc_group_norm_t* d)
{
    if (!d) return SC_ERR_NULL;
    if (d->N < 0 || d->S < 0 || d->C <= 0 || d->G <= 0 || d->C % d->G) return SC_ERR_SHAPE;
    if (!is_wide(d->x_type) || (d->y_type != d->x_type && d->y_type != SC_ELEM_E4M3)) return SC_ERR_UNSUPPORTED;
    if (d->act < SC_ACT_NONE || d->act > SC_ACT_SILU || !(d->eps >= 0.0f) || d->eps > 3e38f) return SC_ERR_UNSUPPORTED;
    if ((int64_t)d->S * d->C >= (int64_t)1 << 31 || (int64_t)d->N * d->S >= (int64_t)1 << 31) return SC_ERR_RANGE;
    if (d->x_sample < 0 || d->x_row < 0) return SC_ERR_SHAPE;
    if (d->y_row < d->C) return SC_ERR_SHAPE;
    if (d->N > 1 && d->S > 0 && d->y_sample < (d->S - 1) * d->y_row + d->C) return SC_ERR_SHAPE;
    if (d->y_type == SC_ELEM_E4M3) {
        if (d->scale_row < ceil_div(d->C, kQBlock)) return SC_ERR_SHAPE;
        if (d->y_row % 16 || d->y_sample % 16) return SC_ERR_UNSUPPORTED;
    }
    return SC_OK;
}

template <int XT, int YT> sc_status_t launch_norm(const sc_group_norm_t* d, const NormArgs& a, hipStream_t stream)
{
    norm_stats_kernel<XT><<<dim3((unsigned)(d->N * d->G)), 256, 0, stream>>>(a);
    if (launched() != SC_OK) return SC_ERR_HIP;
    const int64_t items = (int64_t)d->N * d->S * a.NB;
    const dim3 grid((unsigned)ceil_div(items, 4));
    if (d->act == SC_ACT_RELU) norm_apply_kernel<XT, YT, SC_ACT_RELU><<<grid, 256, 0, stream>>>(a, items);
    else if (d->act == SC_ACT_SILU) norm_apply_kernel<XT, YT, SC_ACT_SILU><<<grid, 256, 0, stream>>>(a, items);
    else norm_apply_kernel<XT, YT, SC_ACT_NONE><<<grid, 256, 0, stream>>>(a, items);
    return launched();
}

template <int XT> sc_status_t launch_norm(const sc_group_norm_t* d, const NormArgs& a, hipStream_t stream)
{
    return d->y_type == SC_ELEM_E4M3 ? launch_norm<XT, SC_ELEM_E4M3>(d, a, stream) : launch_norm<XT, XT>(d, a, stream);
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_group_norm_workspace_size(const sc_group_norm_t* d, size_t* bytes)
{
    if (!bytes) return SC_ERR_NULL;
    const sc_status_t st = check_norm(d);
    if (st != SC_OK) return st;
    *bytes = (size_t)d->N * d->G * sizeof(float2);
    return SC_OK;
}

extern "C" sc_status_t sparse_conv_group_norm(const sc_group_norm_t* d, const void* x, const float* gamma, const float* beta,
                                              void* y, float* y_scale, void* workspace_dev, size_t workspace_bytes, void* stream)
{
    const sc_status_t st = check_norm(d);
    if (st != SC_OK) return st;
    if (d->N == 0 || d->S == 0) return SC_OK;
    const bool codes = d->y_type == SC_ELEM_E4M3;
    if (!x || !y || (codes && !y_scale)) return SC_ERR_NULL;
    if (!aligned(x, elem_bytes(d->x_type)) || !aligned(y, codes ? 16 : elem_bytes(d->y_type)) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(y_scale, 4))
        return SC_ERR_UNSUPPORTED;
    const size_t need = (size_t)d->N * d->G * sizeof(float2);
    if (need && (!workspace_dev || workspace_bytes < need || !aligned(workspace_dev, 16))) return SC_ERR_WORKSPACE;
    NormArgs a;
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.ys = y_scale;
    a.stats = static_cast<float2*>(workspace_dev);
    a.S = d->S; a.C = d->C; a.G = d->G; a.Cg = d->C / d->G; a.NB = (int)ceil_div(d->C, kQBlock);
    a.eps = d->eps;
    a.x_sample = d->x_sample; a.x_row = d->x_row; a.y_sample = d->y_sample; a.y_row = d->y_row; a.s_row = d->scale_row;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (d->x_type) {
        case SC_ELEM_F32: return launch_norm<SC_ELEM_F32>(d, a, s);
        case SC_ELEM_F16: return launch_norm<SC_ELEM_F16>(d, a, s);
        default: return launch_norm<SC_ELEM_BF16>(d, a, s);
    }
}
