// Products in blocks (sparse_conv_matmul_blocks) and grouped by expert (sparse_conv_matmul_grouped).
#include "op_common.h"

namespace sc {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

struct MatmulArgs {
    const uint8_t* a;
    const uint8_t* b;
    const float* as;
    const float* bs;
    const float* bias;
    const int32_t* index;
    const int32_t* offsets;
    void* y;
    int M, N, E, a_rows;
    int kbytes;                              // bytes of a row that count
    int64_t a_row, b_row, b_expert;          // bytes
    int64_t y_row;                           // elements
    int64_t as_row, bs_row, bs_expert;
    int act;
};

// The 16 bytes of a row that begin at `at`, zeros behind the end of the row.
__device__ __forceinline__ v4i row_chunk(const uint8_t* row, int at, int kbytes)
{
    v4i v = {0, 0, 0, 0};
    if (!row || at >= kbytes) return v;
    v = *reinterpret_cast<const v4i*>(row + at);
    const int have = kbytes - at;
    if (have < 16)
        for (int i = 0; i < 4; ++i) {
            const int h = have - 4 * i;
            v[i] = h <= 0 ? 0 : h >= 4 ? v[i] : v[i] & ((1 << (8 * h)) - 1);
        }
    return v;
}

// Eight codes as 16-bit floats (which hold every code).
__device__ __forceinline__ v8h widen8(int lo, int hi)
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ float act_of(float z, int act)
{
    return act == SC_ACT_RELU ? activate<SC_ACT_RELU>(z) : act == SC_ACT_SILU ? activate<SC_ACT_SILU>(z) : z;
}

// Rows of group e: [lo, hi), whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int e, int M, int& lo, int& hi)
{
    lo = min(max(offsets[e], 0), M);
    hi = max(lo, min(max(offsets[e + 1], 0), M));
}

// 64 rows x 64 columns of y per workgroup, four waves of 32 x 32.  The weights are the first operand of the matrix
// instructions, so that a lane's sums belong to one row of y (lane % 16) and four columns (lane / 16).
template <int AT, int YT, bool GROUPED> __global__ __launch_bounds__(256) void matmul_kernel(MatmulArgs p)
{
    constexpr int P = 144;                   // bytes of a staged row: 128 and 16 to spread the banks
    __shared__ __align__(16) uint8_t As[64 * P], Bs[64 * P];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int e = 0, lo = 0, hi = p.M, tile = blockIdx.x;
    if constexpr (GROUPED) {
        for (e = 0; e < p.E; ++e) {
            group_rows(p.offsets, e, p.M, lo, hi);
            const int t = (hi - lo + 63) / 64;
            if (tile < t) break;
            tile -= t;
        }
        if (e == p.E) return;
    }
    const int m0 = lo + tile * 64, n0 = blockIdx.y * 64;
    const uint8_t* arow[2];
    const uint8_t* brow[2];
    for (int i = 0; i < 2; ++i) {
        const int r = (tid >> 3) + 32 * i;
        int m = m0 + r;
        arow[i] = nullptr;
        if (m < hi) {
            if (GROUPED && p.index) m = p.index[m];
            if (m >= 0 && m < p.a_rows) arow[i] = p.a + m * p.a_row;
        }
        brow[i] = n0 + r < p.N ? p.b + e * p.b_expert + (n0 + r) * p.b_row : nullptr;
    }
    const int wm = (wave & 1) * 32, wn = (wave >> 1) * 32;
    const float* as[2] = {nullptr, nullptr};
    const float* bs = nullptr;
    if constexpr (AT == SC_ELEM_E4M3) {
        for (int j = 0; j < 2; ++j) {
            int m = min(m0 + wm + 16 * j + (lane & 15), hi - 1);
            if (GROUPED && p.index) m = min(max(p.index[m], 0), p.a_rows - 1);
            as[j] = p.as + m * p.as_row;
        }
        bs = p.bs + e * p.bs_expert + n0 / kQBlock * p.bs_row;
    }
    v4f acc[2][2] = {};
    for (int kb = 0, k = 0; k < p.kbytes; ++kb, k += 128) {
        __syncthreads();
        for (int i = 0; i < 2; ++i) {
            const int o = ((tid >> 3) + 32 * i) * P + (tid & 7) * 16;
            *reinterpret_cast<v4i*>(As + o) = row_chunk(arow[i], k + (tid & 7) * 16, p.kbytes);
            *reinterpret_cast<v4i*>(Bs + o) = row_chunk(brow[i], k + (tid & 7) * 16, p.kbytes);
        }
        __syncthreads();
        v4i fa[2][2], fb[2][2];
        for (int j = 0; j < 2; ++j)
            for (int h = 0; h < 2; ++h) {
                fa[j][h] = *reinterpret_cast<const v4i*>(As + (wm + 16 * j + (lane & 15)) * P + (lane >> 4) * 32 + h * 16);
                fb[j][h] = *reinterpret_cast<const v4i*>(Bs + (wn + 16 * j + (lane & 15)) * P + (lane >> 4) * 32 + h * 16);
            }
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j) {
                if constexpr (AT == SC_ELEM_E4M3 && YT == SC_ELEM_F32) {
                    v4f d = {0, 0, 0, 0};
                    for (int h = 0; h < 2; ++h)
                        for (int q = 0; q < 2; ++q)
                            d = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8(fb[i][h][2 * q], fb[i][h][2 * q + 1]), widen8(fa[j][h][2 * q], fa[j][h][2 * q + 1]), d, 0, 0, 0);
                    const float s = as[j][kb] * bs[kb];
                    for (int v = 0; v < 4; ++v) acc[i][j][v] += s * d[v];
                } else if constexpr (AT == SC_ELEM_E4M3) {
                    const v8i x = __builtin_shufflevector(fb[i][0], fb[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
                    const v8i w = __builtin_shufflevector(fa[j][0], fa[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
                    const v4f d = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, w, v4f{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
                    const float s = as[j][kb] * bs[kb];
                    for (int v = 0; v < 4; ++v) acc[i][j][v] += s * d[v];
                } else {
                    for (int h = 0; h < 2; ++h)
                        if constexpr (AT == SC_ELEM_F16)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, fb[i][h]), __builtin_bit_cast(v8h, fa[j][h]), acc[i][j], 0, 0, 0);
                        else
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8b, fb[i][h]), __builtin_bit_cast(v8b, fa[j][h]), acc[i][j], 0, 0, 0);
                }
            }
    }
    for (int j = 0; j < 2; ++j) {
        const int m = m0 + wm + 16 * j + (lane & 15);
        if (m >= hi) continue;
        Elem<YT>* y = static_cast<Elem<YT>*>(p.y) + m * p.y_row;
        for (int i = 0; i < 2; ++i)
            for (int v = 0; v < 4; ++v) {
                const int n = n0 + wn + 16 * i + (lane >> 4) * 4 + v;
                if (n < p.N) y[n] = (Elem<YT>)act_of(acc[i][j][v] + (p.bias ? p.bias[(int64_t)e * p.N + n] : 0.0f), p.act);
            }
    }
}

template <int AT, int YT, bool GROUPED> sc_status_t launch(const MatmulArgs& p, hipStream_t stream)
{
    const int64_t tiles = ceil_div(p.M, 64) + (GROUPED ? p.E : 0);
    matmul_kernel<AT, YT, GROUPED><<<dim3((unsigned)tiles, (unsigned)ceil_div(p.N, 64)), 256, 0, stream>>>(p);
    return launched();
}

constexpr int64_t kMaxRowBytes = (int64_t)1 << 22;

sc_status_t check_blocks(const sc_matmul_blocks_t* d)
{
    if (!d) return SC_ERR_NULL;
    const int64_t KB = ceil_div(d->K, kQBlock);
    if (d->M < 0 || d->N <= 0 || d->K <= 0 || d->a_row < d->K || d->b_row < d->K || d->y_row < d->N || d->a_scale_row < KB || d->b_scale_row < KB)
        return SC_ERR_SHAPE;
    if (!is_wide(d->y_type) || d->act < SC_ACT_NONE || d->act > SC_ACT_SILU || d->a_row % 16 || d->b_row % 16) return SC_ERR_UNSUPPORTED;
    if (d->a_row >= kMaxRowBytes || d->b_row >= kMaxRowBytes || d->y_row * 4 * 256 >= (int64_t)1 << 31) return SC_ERR_RANGE;
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
    if (d->b_expert < (d->N - 1) * d->b_row + d->K && d->E > 1) return SC_ERR_SHAPE;
    if (codes && (d->a_scale_row < KB || d->b_scale_row < KB || (d->E > 1 && d->b_scale_expert < ceil_div(d->N, kQBlock) * KB))) return SC_ERR_SHAPE;
    if (d->act < SC_ACT_NONE || d->act > SC_ACT_SILU || d->a_row * e % 16 || d->b_row * e % 16 || d->b_expert * e % 16) return SC_ERR_UNSUPPORTED;
    if (d->a_row * e >= kMaxRowBytes || d->b_row * e >= kMaxRowBytes || d->y_row * 4 * 256 >= (int64_t)1 << 31) return SC_ERR_RANGE;
    return SC_OK;
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
    MatmulArgs p{};
    p.a = static_cast<const uint8_t*>(a); p.b = static_cast<const uint8_t*>(b); p.as = a_scale; p.bs = b_scale; p.bias = bias; p.y = y;
    p.M = d->M; p.N = d->N; p.E = 1; p.a_rows = d->M; p.kbytes = d->K;
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
    MatmulArgs p{};
    p.a = static_cast<const uint8_t*>(a); p.b = static_cast<const uint8_t*>(b); p.as = a_scale; p.bs = b_scale; p.bias = bias;
    p.index = index; p.offsets = offsets; p.y = y;
    p.M = d->M; p.N = d->N; p.E = d->E; p.a_rows = d->a_rows; p.kbytes = d->K * e;
    p.a_row = d->a_row * e; p.b_row = d->b_row * e; p.b_expert = d->b_expert * e; p.y_row = d->y_row;
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
