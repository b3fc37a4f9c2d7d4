// Group norm with an activation, channels last (sparse_conv_group_norm).
//
// Bound by memory: x read once (twice where it does not fit a workgroup), y written once.  Two forms:
//
//   one launch   a workgroup holds whole groups of one sample in its registers, all positions of them: mean, then the squared
//                deviations from it, then the result, with no second look at memory.  Taken where that fits (norm_resident).
//   two launches statistics of stretches of positions (each: mean and sum of squared deviations, put together pairwise, never as
//                a difference of large sums), then the result, whose workgroups first put their sample's stretches together.
//                x comes from the last-level cache the second time where it fits there (256 MB).
#include "op_common.h"

#include <algorithm>

namespace sc {
namespace {

constexpr int kThreads = 256;                // of a workgroup of the two-launch form
constexpr int kMaxStretches = 64;            // stretches of positions of a sample

struct NormArgs {
    const void* x;
    const float* gamma;
    const float* beta;
    void* y;
    float* ys;
    float2* stats;                           // [N][G][stretches][parts] mean, sum of squared deviations
    int N, S, C, G, Cg;
    int seg, segs, parts;                    // channels of a statistics workgroup, segments of C, segments of one group (1: whole groups)
    int len, stretches;                      // positions of a stretch, stretches of a sample
    int rows;                                // positions of a workgroup of the second launch
    float eps;
    int64_t x_sample, x_row, y_sample, y_row, s_row;
};

// Two sets of values as one: (n, mean, m2) takes in (n2, mean2, m2_2).
__device__ __forceinline__ void join(float& n, float& mean, float& m2, float n2, float mean2, float m2_2)
{
    const float all = n + n2, d = mean2 - mean, share = all > 0.0f ? n2 / all : 0.0f;
    mean += d * share;
    m2 += m2_2 + d * d * n * share;
    n = all;
}

// y of V neighbouring channels of one position.
template <int ACT, int V>
__device__ __forceinline__ void finish(float* f, const float* mean, const float* inv, const float* gam, const float* bet, int have)
{
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i < have ? activate<ACT>((f[i] - mean[i]) * inv[i] * gam[i] + bet[i]) : 0.0f;
}

// ---------------------------------------------------------------------------------------------------------------------------
// One launch.  TPR lanes side by side cover the channels of a workgroup (16 bytes each, a power of two, LPG of them a group), the
// others of the T lanes the positions; U positions a lane.  A sum over a group is a sum over lanes of a wave by shuffles and one over
// the waves through LDS.
// ---------------------------------------------------------------------------------------------------------------------------
template <int XT, int YT, int ACT, int T, int U> __global__ __launch_bounds__(T) void norm_resident_kernel(NormArgs a, int TPR, int LPG)
{
    constexpr int V = kVec<XT>, W = T / 64;
    __shared__ float red[2][W][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int slabs = a.C / (TPR * V), n = blockIdx.x / slabs, c0 = (blockIdx.x - n * slabs) * TPR * V;
    const int col = threadIdx.x & (TPR - 1), r0 = threadIdx.x / TPR, R = T / TPR, c = c0 + col * V;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + c;
    float gam[V], bet[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        gam[i] = a.gamma ? a.gamma[c + i] : 1.0f;
        bet[i] = a.beta ? a.beta[c + i] : 0.0f;
    }
    v4i raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (r0 + u * R < a.S) raw[u] = load_raw<XT>(x + (r0 + u * R) * a.x_row);
    const float cnt = (float)a.S * (float)a.Cg;
    auto total = [&](float v, int which) {
        for (int o = 1; o < LPG; o <<= 1) v += __shfl_xor(v, o);
        for (int o = TPR; o < 64; o <<= 1) v += __shfl_xor(v, o);
        red[which][wave][lane] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += red[which][w][lane];
        return s;
    };
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (r0 + u * R < a.S) {
            float f[V], part = 0.0f;
            to_floats<XT>(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) part += f[i];
            s += part;
        }
    const float mean = total(s, 0) / cnt;
    s = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (r0 + u * R < a.S) {
            float f[V], part = 0.0f;
            to_floats<XT>(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) part += (f[i] - mean) * (f[i] - mean);
            s += part;
        }
    const float inv = 1.0f / sqrtf(total(s, 1) / cnt + a.eps);
    float means[V], invs[V];
#pragma unroll
    for (int i = 0; i < V; ++i) means[i] = mean, invs[i] = inv;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int pos = r0 + u * R;
        if (pos >= a.S) continue;            // (a position's lanes go on or leave together: the shuffles below stay inside it)
        float f[V];
        to_floats<XT>(raw[u], f);
        finish<ACT, V>(f, means, invs, gam, bet, V);
        Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + n * a.y_sample + pos * a.y_row + c;
        if constexpr (YT == SC_ELEM_E4M3) {
            constexpr int L = kQBlock / V;
            float amax = kAmaxFloor;
#pragma unroll
            for (int i = 0; i < V; ++i) amax = fmaxf(amax, fabsf(f[i]));
#pragma unroll
            for (int o = L / 2; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
            store_codes<V>(y, f, kCodeMax / amax);
            if (col % L == 0) a.ys[((int64_t)n * a.S + pos) * a.s_row + c / kQBlock] = amax / kCodeMax;
        } else {
            store_vec<YT, V>(y, f, V);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------------
// Two launches, the first: one workgroup per (sample, stretch of positions, segment of channels).  A lane keeps V neighbouring
// channels and takes U positions at a time: their mean, their squared deviations from it, and both joined to what it has.
// ---------------------------------------------------------------------------------------------------------------------------
template <int XT> __global__ __launch_bounds__(kThreads) void norm_stats_kernel(NormArgs a)
{
    constexpr int V = kVec<XT>, U = 8;
    __shared__ float ms[kThreads * V], qs[kThreads * V], ns[kThreads];
    int id = blockIdx.x;
    const int sg = id % a.segs;
    id /= a.segs;
    const int st = id % a.stretches, n = id / a.stretches;
    // (a.parts > 1: a segment is a part of one group; else whole groups)
    const int g0 = a.parts > 1 ? sg / a.parts : sg * (a.seg / a.Cg), part = a.parts > 1 ? sg % a.parts : 0;
    const int c0 = a.parts > 1 ? g0 * a.Cg + part * a.seg : sg * a.seg;
    const int cn = a.parts > 1 ? min(a.seg, a.Cg - part * a.seg) : min(a.seg, a.C - c0);
    const int tpr = (cn + V - 1) / V, R = kThreads / tpr;
    const int r = threadIdx.x / tpr, v = threadIdx.x - r * tpr;
    const int p0 = st * a.len, pn = min(a.len, a.S - p0);
    const int have = min(V, cn - v * V);
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + p0 * a.x_row + c0 + v * V;
    float mean[V] = {}, m2[V] = {}, cnt = 0.0f;
    if (r < R) {
        int p = r;
        for (; p + (U - 1) * R < pn; p += U * R) {
            v4i raw[U];
            if (have == V) {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = load_raw<XT>(x + (p + u * R) * a.x_row);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) raw[u] = load_raw_part<XT>(x + (p + u * R) * a.x_row, have);
            }
            const float share = (float)U / (cnt + (float)U);
            float sum[V] = {}, sq[V] = {};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[V];
                to_floats<XT>(raw[u], f);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] += f[i];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] *= 1.0f / U;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[V];
                to_floats<XT>(raw[u], f);
#pragma unroll
                for (int i = 0; i < V; ++i) sq[i] += (f[i] - sum[i]) * (f[i] - sum[i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = sum[i] - mean[i];
                mean[i] += d * share;
                m2[i] += sq[i] + d * d * cnt * share;
            }
            cnt += (float)U;
        }
        for (; p < pn; p += R) {
            float f[V];
            to_floats<XT>(have == V ? load_raw<XT>(x + p * a.x_row) : load_raw_part<XT>(x + p * a.x_row, have), f);
            cnt += 1.0f;
            const float share = 1.0f / cnt;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = f[i] - mean[i];
                mean[i] += d * share;
                m2[i] += d * (f[i] - mean[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ms[threadIdx.x * V + i] = mean[i];
        qs[threadIdx.x * V + i] = m2[i];
    }
    ns[threadIdx.x] = r < R ? cnt : 0.0f;
    __syncthreads();
    // Sixteen lanes put a group together: the mean of the means, then the deviations around it.
    const int groups = a.parts > 1 ? 1 : cn / a.Cg, gc = a.parts > 1 ? cn : a.Cg;
    const int sub = threadIdx.x >> 4, sl = threadIdx.x & 15;
    const float total = (float)pn * (float)gc;
    for (int g = sub; g < groups; g += kThreads / 16) {
        float s = 0.0f;
        for (int i = sl; i < R * gc; i += 16) {
            const int rr = i / gc, cc = g * gc + (i - rr * gc);
            s += ns[rr * tpr + cc / V] * ms[rr * tpr * V + cc];
        }
        for (int o = 8; o; o >>= 1) s += __shfl_xor(s, o);
        const float m = s / total;
        float q = 0.0f;
        for (int i = sl; i < R * gc; i += 16) {
            const int rr = i / gc, cc = g * gc + (i - rr * gc);
            const float d = ms[rr * tpr * V + cc] - m;
            q += qs[rr * tpr * V + cc] + ns[rr * tpr + cc / V] * d * d;
        }
        for (int o = 8; o; o >>= 1) q += __shfl_xor(q, o);
        if (sl == 0) a.stats[(((int64_t)n * a.G + g0 + g) * a.stretches + st) * a.parts + part] = make_float2(m, q);
    }
}

// The second: one workgroup per (sample, a.rows positions, up to kThreads * V channels).  Codes: a row's lanes are padded to whole
// blocks of 128 channels, so that a block's lanes are neighbours in one wave.
template <int XT, int YT, int ACT> __global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a, int wide, int wides, int chunks)
{
    constexpr int V = kVec<XT>, U = 4, L = kQBlock / V;
    constexpr bool CODES = YT == SC_ELEM_E4M3;
    extern __shared__ float2 gs[];           // mean, 1 / spread of the groups of this workgroup
    int id = blockIdx.x;
    const int sg = id % wides;
    id /= wides;
    const int ch = id % chunks, n = id / chunks;
    const int c0 = sg * wide, cn = min(wide, a.C - c0);
    const int g0 = c0 / a.Cg, groups = (c0 + cn - 1) / a.Cg - g0 + 1;
    const int sub = threadIdx.x >> 4, sl = threadIdx.x & 15, per = a.stretches * a.parts;
    for (int g = sub; g < groups; g += kThreads / 16) {
        float cnt = 0.0f, mean = 0.0f, m2 = 0.0f;
        const float2* st = a.stats + ((int64_t)n * a.G + g0 + g) * per;
        for (int i = sl; i < per; i += 16) {
            const int s = i / a.parts, part = i - s * a.parts;
            const int chans = a.parts > 1 ? min(a.seg, a.Cg - part * a.seg) : a.Cg;
            const float2 v = st[i];
            join(cnt, mean, m2, (float)min(a.len, a.S - s * a.len) * (float)chans, v.x, v.y);
        }
        for (int o = 8; o; o >>= 1) {
            const float n2 = __shfl_xor(cnt, o), mean2 = __shfl_xor(mean, o), q2 = __shfl_xor(m2, o);
            if (sl & o) {                    // (both lanes of a pair join in the same order)
                float n1 = n2, me = mean2, q = q2;
                join(n1, me, q, cnt, mean, m2);
                cnt = n1, mean = me, m2 = q;
            } else {
                join(cnt, mean, m2, n2, mean2, q2);
            }
        }
        if (sl == 0) gs[g] = make_float2(mean, 1.0f / sqrtf(m2 / cnt + a.eps));
    }
    __syncthreads();
    const int tpr = CODES ? (cn + kQBlock - 1) / kQBlock * L : (cn + V - 1) / V;
    const int R = kThreads / tpr, r = threadIdx.x / tpr, v = threadIdx.x - r * tpr;
    const int have = min(V, cn - v * V), c = c0 + v * V;
    float mean[V], inv[V], gam[V], bet[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        mean[i] = bet[i] = 0.0f, inv[i] = gam[i] = 1.0f;
        if (i < have) {
            const float2 s = gs[(c + i) / a.Cg - g0];
            mean[i] = s.x, inv[i] = s.y;
            if (a.gamma) gam[i] = a.gamma[c + i];
            if (a.beta) bet[i] = a.beta[c + i];
        }
    }
    if (r >= R) return;
    const int p0 = ch * a.rows, p1 = min(a.S, p0 + a.rows);
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + c;
    Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + n * a.y_sample + c;
    for (int p = p0 + r; p < p1; p += U * R) {
        v4i raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = v4i{0, 0, 0, 0};
            if (p + u * R < p1) raw[u] = have == V ? load_raw<XT>(x + (p + u * R) * a.x_row) : load_raw_part<XT>(x + (p + u * R) * a.x_row, have);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = p + u * R;
            if (pos >= p1) break;            // (the lanes of a position leave together)
            float f[V];
            to_floats<XT>(raw[u], f);
            finish<ACT, V>(f, mean, inv, gam, bet, have);
            if constexpr (CODES) {
                float amax = kAmaxFloor;
#pragma unroll
                for (int i = 0; i < V; ++i) amax = fmaxf(amax, fabsf(f[i]));
#pragma unroll
                for (int o = L / 2; o; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
                if (c < ((a.C + 15) & ~15)) store_codes<V>(y + pos * a.y_row, f, kCodeMax / amax);
                if (v % L == 0) a.ys[((int64_t)n * a.S + pos) * a.s_row + c / kQBlock] = amax / kCodeMax;
            } else {
                store_vec<YT, V>(y + pos * a.y_row, f, have);
            }
        }
    }
}

bool pow2(int v) { return v > 0 && (v & (v - 1)) == 0; }

struct NormShape {
    int TPR, LPG, T, U;                      // one launch (TPR = 0: two)
    int seg, segs, parts, len, stretches;    // the statistics
    int wide, wides, rows, chunks;           // the result
    size_t bytes;
};

// One launch: groups of a power of two of 16-byte lanes, channels of a workgroup whole 128-byte lines (codes: whole blocks) where
// C allows it, and all positions of them in 16 vectors a lane of 512.
bool norm_resident(const sc_group_norm_t* d, NormShape* s)
{
    const int V = 16 / elem_bytes(d->x_type), Cg = d->C / d->G;
    if (Cg % V || !pow2(Cg / V) || Cg / V > 64) return false;
    const int LPG = Cg / V, line = d->y_type == SC_ELEM_E4M3 ? kQBlock / V : 8;
    int TPR = LPG;
    while (TPR < line && d->C % (2 * TPR * V) == 0) TPR *= 2;
    if (TPR > 64 || (d->y_type == SC_ELEM_E4M3 && TPR % line)) return false;
    const int64_t vectors = (int64_t)d->S * TPR;
    if (vectors > 512 * 16) return false;
    s->TPR = TPR;
    s->LPG = LPG;
    s->T = vectors <= 256 * 4 ? 256 : 512;
    s->U = vectors <= s->T * 4 ? 4 : 16;
    return true;
}

NormShape norm_shape(const sc_group_norm_t* d)
{
    NormShape s{};
    if (d->N == 0 || d->S == 0 || norm_resident(d, &s)) return s;
    const int V = 16 / elem_bytes(d->x_type), Cg = d->C / d->G, most = kThreads * V;
    if (Cg <= most) {
        s.seg = std::min(d->G, most / Cg) * Cg;
        s.parts = 1;
        s.segs = (int)ceil_div(d->C, s.seg);
    } else {
        s.seg = most;
        s.parts = (int)ceil_div(Cg, most);
        s.segs = d->G * s.parts;
    }
    // Four workgroups a compute unit for both launches, no stretch under eight vectors a lane.
    const int R = std::max<int>(1, kThreads / (int)ceil_div(std::min(s.seg, d->C), V));
    const int64_t want = std::max<int64_t>(1, 1024 / ((int64_t)d->N * s.segs));
    s.stretches = (int)std::min<int64_t>({want, kMaxStretches, ceil_div(d->S, 8 * R)});
    s.len = (int)ceil_div(d->S, s.stretches);
    s.stretches = (int)ceil_div(d->S, s.len);
    s.wide = std::min(most, d->C);
    s.wides = (int)ceil_div(d->C, s.wide);
    const int R2 = std::max<int>(1, kThreads / (int)ceil_div(s.wide, V));
    const int64_t want2 = std::max<int64_t>(1, 2048 / ((int64_t)d->N * s.wides));
    s.rows = (int)std::max<int64_t>(ceil_div(d->S, want2), 4 * R2);
    s.chunks = (int)ceil_div(d->S, s.rows);
    s.bytes = (size_t)d->N * d->G * s.stretches * s.parts * sizeof(float2);
    return s;
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

template <int XT, int YT, int ACT> sc_status_t launch_norm(const sc_group_norm_t* d, const NormShape& s, const NormArgs& a, hipStream_t stream)
{
    if (s.TPR) {
        const int64_t blocks = (int64_t)d->N * (d->C / (s.TPR * kVec<XT>));
        if (blocks * s.T >= (int64_t)1 << 32) return SC_ERR_RANGE;
        const dim3 grid((unsigned)blocks);
        if (s.T == 256) norm_resident_kernel<XT, YT, ACT, 256, 4><<<grid, 256, 0, stream>>>(a, s.TPR, s.LPG);
        else if (s.U == 4) norm_resident_kernel<XT, YT, ACT, 512, 4><<<grid, 512, 0, stream>>>(a, s.TPR, s.LPG);
        else norm_resident_kernel<XT, YT, ACT, 512, 16><<<grid, 512, 0, stream>>>(a, s.TPR, s.LPG);
        return launched();
    }
    const int64_t first = (int64_t)d->N * s.segs * s.stretches, second = (int64_t)d->N * s.wides * s.chunks;
    if (std::max(first, second) * kThreads >= (int64_t)1 << 32) return SC_ERR_RANGE;
    norm_stats_kernel<XT><<<dim3((unsigned)first), kThreads, 0, stream>>>(a);
    if (launched() != SC_OK) return SC_ERR_HIP;
    const size_t lds = (size_t)std::min<int64_t>(d->G, ceil_div(s.wide, a.Cg) + 1) * sizeof(float2);
    norm_apply_kernel<XT, YT, ACT><<<dim3((unsigned)second), kThreads, lds, stream>>>(a, s.wide, s.wides, s.chunks);
    return launched();
}

template <int XT, int YT> sc_status_t launch_norm(const sc_group_norm_t* d, const NormShape& s, const NormArgs& a, hipStream_t stream)
{
    return d->act == SC_ACT_RELU   ? launch_norm<XT, YT, SC_ACT_RELU>(d, s, a, stream)
           : d->act == SC_ACT_SILU ? launch_norm<XT, YT, SC_ACT_SILU>(d, s, a, stream)
                                   : launch_norm<XT, YT, SC_ACT_NONE>(d, s, a, stream);
}

template <int XT> sc_status_t launch_norm(const sc_group_norm_t* d, const NormShape& s, const NormArgs& a, hipStream_t stream)
{
    return d->y_type == SC_ELEM_E4M3 ? launch_norm<XT, SC_ELEM_E4M3>(d, s, a, stream) : launch_norm<XT, XT>(d, s, a, stream);
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_group_norm_workspace_size(const sc_group_norm_t* d, size_t* bytes)
{
    if (!bytes) return SC_ERR_NULL;
    const sc_status_t st = check_norm(d);
    if (st != SC_OK) return st;
    *bytes = norm_shape(d).bytes;
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
    const NormShape shape = norm_shape(d);
    if (shape.bytes && (!workspace_dev || workspace_bytes < shape.bytes || !aligned(workspace_dev, 16))) return SC_ERR_WORKSPACE;
    NormArgs a;
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.ys = y_scale;
    a.stats = static_cast<float2*>(workspace_dev);
    a.N = d->N; a.S = d->S; a.C = d->C; a.G = d->G; a.Cg = d->C / d->G;
    a.seg = shape.seg; a.segs = shape.segs; a.parts = shape.parts; a.len = shape.len; a.stretches = shape.stretches; a.rows = shape.rows;
    a.eps = d->eps;
    a.x_sample = d->x_sample; a.x_row = d->x_row; a.y_sample = d->y_sample; a.y_row = d->y_row; a.s_row = d->scale_row;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (d->x_type) {
        case SC_ELEM_F32: return launch_norm<SC_ELEM_F32>(d, shape, a, s);
        case SC_ELEM_F16: return launch_norm<SC_ELEM_F16>(d, shape, a, s);
        default: return launch_norm<SC_ELEM_BF16>(d, shape, a, s);
    }
}
