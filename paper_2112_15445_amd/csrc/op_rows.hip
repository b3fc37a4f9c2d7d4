// Rows out to their places and back (sparse_conv_gather_rows, sparse_conv_combine_rows and its gradients).
//
// All of them are bound by memory: sixteen bytes a lane (of x), lanes along a row, several rows under way at once.  What is read once goes past
// the caches, and so do results of more than 32 MiB (8192 x 2 rows of 4096 bf16 back with a residual 52 -> 47 us, 5.7 TB/s; 4096 x 8 rows of 2048 back 35 -> 29, out 39 -> 36).
// Smaller ones stay in them for the call behind (us, through the caches and past them; rows of bf16, out alone and with a product by expert of 1024 columns behind: 8 x 2 of
// 2048 3.4 and 3.5, 11.2 and 12.2; 256 x 2 3.6 and 3.6, 12.8 and 15.1; 2048 x 2 6.1 and 5.9, 38 and 42; back alone and with a quantiser behind: 8192 of 2048 24.6 and 25.5, 35 and
// 38; 4096 of 4096 25.9 and 25.2, 36.6 and 37.0).  Of larger ones less is left there than it costs: out with a quantiser 64 MiB 22 and 20, 39 and 41, 128 MiB 43 and 39, 77 and 75;
// back 64 MiB 54 and 46, 71 and 72.  (A product that reads its rows again for every tile of columns would have 64 MiB there, 70 and 78.)
#include "op_common.h"

#include <algorithm>
#include <type_traits>

namespace sc {
namespace {

constexpr int kRowThreads = 256;
constexpr int64_t kKept = 32 << 20;          // bytes of a result that stay in the caches

struct GatherArgs {
    const uint8_t* x;
    const int32_t* index;
    uint8_t* y;
    int M, rows, chunks, lanes, bytes;       // 16-byte chunks of a row, lanes of a row (a power of two), bytes of a row
    int64_t x_row, y_row;                    // bytes
};

__device__ __forceinline__ v4i chunk_of(const uint8_t* row, int have)
{
    v4i v = {0, 0, 0, 0};
    if (have >= 16) __builtin_memcpy(&v, row, 16);
    else {
        uint8_t b[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) b[i] = row[min(i, have - 1)];
        __builtin_memcpy(&v, b, 16);
    }
    return v;
}
template <bool PAST> __device__ __forceinline__ void put_chunk(uint8_t* row, v4i v, int have)
{
    typedef int any4i __attribute__((ext_vector_type(4), aligned(1)));
    if (have >= 16) {
        if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<any4i*>(row));
        else *reinterpret_cast<any4i*>(row) = v;
    } else {
        uint8_t b[16];
        __builtin_memcpy(b, &v, 16);
#pragma unroll
        for (int i = 0; i < 15; ++i)
            if (i < have) row[i] = b[i];
    }
}

// U rows a lane under way at once.
template <int U, bool PAST> __global__ __launch_bounds__(kRowThreads) void gather_rows_kernel(GatherArgs a)
{
    const int per = kRowThreads / a.lanes, lane = threadIdx.x & (a.lanes - 1);
    const int64_t first = (int64_t)blockIdx.x * (per * U) + threadIdx.x / a.lanes;
    int from[U];
#pragma unroll
    for (int u = 0; u < U; ++u) from[u] = first + u * per < a.M ? a.index[first + u * per] : -1;
    for (int c = lane; c < a.chunks; c += a.lanes) {
        const int have = a.bytes - c * 16;
        v4i v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            v[u] = v4i{0, 0, 0, 0};
            if ((uint32_t)from[u] < (uint32_t)a.rows) v[u] = chunk_of(a.x + from[u] * a.x_row + c * 16, have);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (first + u * per < a.M) put_chunk<PAST>(a.y + (first + u * per) * a.y_row + c * 16, v[u], have);
    }
}

struct CombineArgs {
    const void* x;
    const int32_t* position;
    const float* weights;
    const void* residual;
    void* y;
    const void* dy;
    void* dx;
    float* dweights;
    int T, top, C, rows, lanes;
    int64_t x_row, y_row, residual_row, dx_row;
};

// V values that are whole, past the caches or through them.  (The choice is the kernel's: of two stores behind a branch the compiler makes one, through the caches.)
template <int ET, bool PAST, int V> __device__ __forceinline__ void put_values(Elem<ET>* y, const float (&f)[V])
{
    if constexpr (PAST) store_once<ET, V>(y, f);
    else store_values<ET, V>(y, V, f);
}

// y[t] = residual[t] + sum over j of weights[t,j] x[position[t,j]], in the order of j, in 32 bits; kSlots rows are read together.
constexpr int kSlots = 4;
template <int XT, int YT, bool PAST> __global__ __launch_bounds__(kRowThreads) void combine_rows_kernel(CombineArgs a)
{
    constexpr int V = kVec<XT>;
    const int per = kRowThreads / a.lanes, lane = threadIdx.x & (a.lanes - 1);
    const int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / a.lanes;
    if (t >= a.T) return;
    const int32_t* position = a.position + t * a.top;
    const float* weights = a.weights ? a.weights + t * a.top : nullptr;
    // (whole: sixteen bytes of x; a branch on that inside would have every load wait for the one before it: 47 -> 61 us)
    auto columns = [&](int c, auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        const int have = WHOLE ? V : a.C - c;
        float sum[V] = {};
        if (a.residual) load_values<YT, V>(static_cast<const Elem<YT>*>(a.residual) + t * a.residual_row + c, have, sum);
        for (int j0 = 0; j0 < a.top; j0 += kSlots) {
            int p[kSlots];
            v4i raw[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                p[j] = position[min(j0 + j, a.top - 1)];
                if (j0 + j >= a.top) p[j] = -1;
            }
#pragma unroll
            for (int j = 0; j < kSlots; ++j)
                if ((uint32_t)p[j] < (uint32_t)a.rows) {
                    const Elem<XT>* row = static_cast<const Elem<XT>*>(a.x) + p[j] * a.x_row + c;
                    if constexpr (WHOLE) raw[j] = load_raw_once<XT>(row);
                    else raw[j] = load_raw_part<XT>(row, have);
                }
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                if ((uint32_t)p[j] >= (uint32_t)a.rows) continue;
                const float w = weights ? weights[j0 + j] : 1.0f;
                float f[V];
                to_floats<XT>(raw[j], f);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] = fmaf(w, f[i], sum[i]);
            }
        }
        Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + t * a.y_row + c;
        if constexpr (WHOLE) put_values<YT, PAST>(y, sum);
        else store_values<YT, V>(y, have, sum);
    };
    int c = lane * V;
    for (; c + V <= a.C; c += a.lanes * V) columns(c, std::true_type{});
    if (c < a.C) columns(c, std::false_type{});
}

// dx[position[t,j]] = weights[t,j] dy[t], dweights[t,j] = sum of dy[t] x[position[t,j]]: L lanes a token (16 or 64, or the workgroup's four waves), kSlots slots at a
// time, whose rows are read together (a slot without a row reads row 0 and drops it, so that no load waits behind a branch).
template <int XT, int YT, int L, bool DX, bool DW, bool PAST> __global__ __launch_bounds__(kRowThreads) void combine_gradient_kernel(CombineArgs a)
{
    constexpr int V = kVec<XT>, W = kRowThreads / 64;
    __shared__ float part[L == kRowThreads ? W : 1][L == kRowThreads ? 64 : 1];
    const int per = kRowThreads / L, lane = threadIdx.x & (L - 1);
    const int64_t t = (int64_t)blockIdx.x * per + threadIdx.x / L, token = t < a.T ? t : a.T - 1;      // (lanes without a token follow the last one's)
    const int32_t* position = a.position + token * a.top;
    const Elem<YT>* dy = static_cast<const Elem<YT>*>(a.dy) + token * a.y_row;
    for (int j0 = 0; j0 < a.top; j0 += kSlots) {
        const Elem<XT>* x[kSlots];
        Elem<XT>* dx[kSlots];
        float w[kSlots], dot[kSlots] = {};
        bool real[kSlots];
#pragma unroll
        for (int j = 0; j < kSlots; ++j) {
            const int at = min(j0 + j, a.top - 1), p = position[at];
            real[j] = j0 + j < a.top && (uint32_t)p < (uint32_t)a.rows;
            w[j] = a.weights ? a.weights[token * a.top + at] : 1.0f;
            x[j] = static_cast<const Elem<XT>*>(a.x) + (real[j] ? p : 0) * a.x_row;
            dx[j] = static_cast<Elem<XT>*>(a.dx) + (real[j] ? p : 0) * a.dx_row;
        }
        if (a.rows > 0) {
            int c = lane * V;
            for (; c + V <= a.C; c += L * V) {
                float g[V];
                v4i raw[kSlots];
                load_values<YT, V>(dy + c, V, g);
                if constexpr (DW)
#pragma unroll
                    for (int j = 0; j < kSlots; ++j)
                        if (j == 0 || j0 + j < a.top) raw[j] = load_raw_once<XT>(x[j] + c);
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if (j > 0 && j0 + j >= a.top) break;
                    float f[V];
                    if constexpr (DW) {
                        to_floats<XT>(raw[j], f);
#pragma unroll
                        for (int i = 0; i < V; ++i) dot[j] = fmaf(g[i], f[i], dot[j]);
                    }
                    if constexpr (DX) {
#pragma unroll
                        for (int i = 0; i < V; ++i) f[i] = g[i] * w[j];
                        if (real[j] && t < a.T) put_values<XT, PAST>(dx[j] + c, f);
                    }
                }
            }
            if (c < a.C) {                   // the last columns, fewer than V
                const int have = a.C - c;
                float g[V];
                load_values<YT, V>(dy + c, have, g);
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if (!real[j]) continue;
                    float f[V];
                    if constexpr (DW) {
                        load_values<XT, V>(x[j] + c, have, f);
#pragma unroll
                        for (int i = 0; i < V; ++i) dot[j] = fmaf(g[i], f[i], dot[j]);
                    }
                    if constexpr (DX) {
#pragma unroll
                        for (int i = 0; i < V; ++i) f[i] = g[i] * w[j];
                        if (t < a.T) store_values<XT, V>(dx[j] + c, have, f);
                    }
                }
            }
        }
        if constexpr (DW)
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                if (j0 + j >= a.top) break;
                float sum = sum16(dot[j]);
                if constexpr (L > 16) {
                    sum += __shfl_xor(sum, 16);
                    sum += __shfl_xor(sum, 32);
                }
                if (!real[j]) sum = 0.0f;
                if constexpr (L == kRowThreads) {
                    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][j0 + j] = sum;
                } else if (lane == 0 && t < a.T) {
                    a.dweights[t * a.top + j0 + j] = sum;
                }
            }
    }
    if constexpr (DW && L == kRowThreads) {
        __syncthreads();
        if ((int)threadIdx.x < a.top) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) sum += part[w][threadIdx.x];
            a.dweights[t * a.top + threadIdx.x] = sum;
        }
    }
}

// Lanes of a row of n chunks: the power of two that holds them, from 4 to the workgroup.
int lanes_of(int64_t n)
{
    int l = 4;
    while (l < kRowThreads && l < n) l *= 2;
    return l;
}

constexpr int kMaxTable = 1 << 30;

sc_status_t check(const sc_combine_rows_t* d, bool back)
{
    if (!d) return SC_ERR_NULL;
    if (d->T < 0 || d->top <= 0 || d->top > 64 || d->C <= 0 || d->rows < 0 || d->x_row < 0 || (back ? d->y_row < 0 : d->y_row < d->C) || d->residual_row < 0 ||
        (back && d->dx_row < d->C))
        return SC_ERR_SHAPE;
    if (!is_wide(d->x_type) || (d->y_type != d->x_type && d->y_type != SC_ELEM_F32)) return SC_ERR_UNSUPPORTED;
    if ((int64_t)d->T * d->top > kMaxTable || d->C > kMaxTable || d->T > 1 << 23) return SC_ERR_RANGE;
    return SC_OK;
}

CombineArgs args(const sc_combine_rows_t* d, const int32_t* position, const float* weights)
{
    CombineArgs a{};
    a.position = position; a.weights = weights;
    a.T = d->T; a.top = d->top; a.C = d->C; a.rows = d->rows;
    a.x_row = d->x_row; a.y_row = d->y_row; a.residual_row = d->residual_row; a.dx_row = d->dx_row;
    return a;
}

template <int XT, int YT> sc_status_t launch_combine(CombineArgs a, hipStream_t s)
{
    a.lanes = lanes_of(ceil_div(a.C, kVec<XT>));
    const unsigned grid = (unsigned)ceil_div(a.T, kRowThreads / a.lanes);
    if ((int64_t)a.T * a.C * (int64_t)sizeof(Elem<YT>) > kKept) combine_rows_kernel<XT, YT, true><<<grid, kRowThreads, 0, s>>>(a);
    else combine_rows_kernel<XT, YT, false><<<grid, kRowThreads, 0, s>>>(a);
    return launched();
}

// A wave a token up to 64 chunks of a row, and up to 192 with many tokens, where the lanes of a workgroup that have no chunk cost more than the turns of a wave
// (us: 16384 x 2 rows of 128 chunks 42 with 256 lanes and 29 with 64, of 192 chunks 50 and 42, 8192 x 2 of 256 chunks 31 and 33; 64 x 8 of 128 chunks 5.1 and 6.6).
template <int XT, int YT, bool DX, bool DW, bool PAST> sc_status_t launch_gradient_of(const CombineArgs& a, hipStream_t s)
{
    const int64_t chunks = ceil_div(a.C, kVec<XT>);
    if (chunks <= 16) combine_gradient_kernel<XT, YT, 16, DX, DW, PAST><<<(unsigned)ceil_div(a.T, 16), kRowThreads, 0, s>>>(a);
    else if (chunks <= 64 || (chunks <= 192 && a.T >= 1024)) combine_gradient_kernel<XT, YT, 64, DX, DW, PAST><<<(unsigned)ceil_div(a.T, 4), kRowThreads, 0, s>>>(a);
    else combine_gradient_kernel<XT, YT, kRowThreads, DX, DW, PAST><<<(unsigned)a.T, kRowThreads, 0, s>>>(a);
    return launched();
}

template <int XT, int YT> sc_status_t launch_gradient(const CombineArgs& a, hipStream_t s)
{
    if (!a.dx) return launch_gradient_of<XT, YT, false, true, false>(a, s);
    const bool past = std::min<int64_t>(a.rows, (int64_t)a.T * a.top) * a.C * (int64_t)sizeof(Elem<XT>) > kKept;
    if (a.dweights) return past ? launch_gradient_of<XT, YT, true, true, true>(a, s) : launch_gradient_of<XT, YT, true, true, false>(a, s);
    return past ? launch_gradient_of<XT, YT, true, false, true>(a, s) : launch_gradient_of<XT, YT, true, false, false>(a, s);
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_gather_rows(const sc_gather_rows_t* d, const void* x, const int32_t* index, void* y, void* stream)
{
    if (!d) return SC_ERR_NULL;
    if (d->M < 0 || d->C <= 0 || d->rows < 0 || d->x_row < 0 || d->y_row < d->C) return SC_ERR_SHAPE;
    if (!is_wide(d->x_type) && d->x_type != SC_ELEM_E4M3) return SC_ERR_UNSUPPORTED;
    const int e = elem_bytes(d->x_type);
    if (d->M > 1 << 23 || d->C > kMaxTable / 4 || d->x_row >= (int64_t)1 << 32 || d->y_row >= (int64_t)1 << 32) return SC_ERR_RANGE;
    if (d->M == 0) return SC_OK;
    if ((!x && d->rows) || !index || !y) return SC_ERR_NULL;
    if (!aligned(x, e) || !aligned(index, 4) || !aligned(y, e)) return SC_ERR_UNSUPPORTED;
    GatherArgs a;
    a.x = static_cast<const uint8_t*>(x); a.index = index; a.y = static_cast<uint8_t*>(y);
    a.M = d->M; a.rows = d->rows; a.bytes = d->C * e; a.chunks = (int)ceil_div(a.bytes, 16); a.lanes = lanes_of(a.chunks);
    a.x_row = d->x_row * e; a.y_row = d->y_row * e;
    constexpr int U = 2;
    const unsigned grid = (unsigned)ceil_div(a.M, kRowThreads / a.lanes * U);
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if ((int64_t)a.M * a.bytes > kKept) gather_rows_kernel<U, true><<<grid, kRowThreads, 0, s>>>(a);
    else gather_rows_kernel<U, false><<<grid, kRowThreads, 0, s>>>(a);
    return launched();
}

extern "C" sc_status_t sparse_conv_combine_rows(const sc_combine_rows_t* d, const void* x, const int32_t* position, const float* weights, const void* residual,
                                                void* y, void* stream)
{
    const sc_status_t st = check(d, false);
    if (st != SC_OK) return st;
    if (d->T == 0) return SC_OK;
    if ((!x && d->rows) || !position || !y) return SC_ERR_NULL;
    const int xe = elem_bytes(d->x_type), ye = elem_bytes(d->y_type);
    if (!aligned(x, xe) || !aligned(y, ye) || !aligned(residual, ye) || !aligned(position, 4) || !aligned(weights, 4)) return SC_ERR_UNSUPPORTED;
    CombineArgs a = args(d, position, weights);
    a.x = x; a.residual = residual; a.y = y;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = d->y_type == SC_ELEM_F32;
    switch (d->x_type) {
        case SC_ELEM_F32: return launch_combine<SC_ELEM_F32, SC_ELEM_F32>(a, s);
        case SC_ELEM_F16: return f32 ? launch_combine<SC_ELEM_F16, SC_ELEM_F32>(a, s) : launch_combine<SC_ELEM_F16, SC_ELEM_F16>(a, s);
        default: return f32 ? launch_combine<SC_ELEM_BF16, SC_ELEM_F32>(a, s) : launch_combine<SC_ELEM_BF16, SC_ELEM_BF16>(a, s);
    }
}

extern "C" sc_status_t sparse_conv_combine_rows_backward(const sc_combine_rows_t* d, const void* dy, const void* x, const int32_t* position, const float* weights,
                                                         void* dx, float* dweights, void* stream)
{
    const sc_status_t st = check(d, true);
    if (st != SC_OK) return st;
    if (d->T == 0) return SC_OK;
    if (!dy || !position || (dweights && !x && d->rows)) return SC_ERR_NULL;
    const int xe = elem_bytes(d->x_type), ye = elem_bytes(d->y_type);
    if (!aligned(x, xe) || !aligned(dx, xe) || !aligned(dy, ye) || !aligned(position, 4) || !aligned(weights, 4) || !aligned(dweights, 4)) return SC_ERR_UNSUPPORTED;
    if (!dx && !dweights) return SC_OK;
    CombineArgs a = args(d, position, weights);
    a.dy = dy; a.x = x; a.dx = dx; a.dweights = dweights;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = d->y_type == SC_ELEM_F32;
    switch (d->x_type) {
        case SC_ELEM_F32: return launch_gradient<SC_ELEM_F32, SC_ELEM_F32>(a, s);
        case SC_ELEM_F16: return f32 ? launch_gradient<SC_ELEM_F16, SC_ELEM_F32>(a, s) : launch_gradient<SC_ELEM_F16, SC_ELEM_F16>(a, s);
        default: return f32 ? launch_gradient<SC_ELEM_BF16, SC_ELEM_F32>(a, s) : launch_gradient<SC_ELEM_BF16, SC_ELEM_BF16>(a, s);
    }
}
