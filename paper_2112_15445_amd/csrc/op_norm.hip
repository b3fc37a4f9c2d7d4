// Group norm with an activation, channels last (sparse_conv_group_norm).
//
// Bound by memory: x read once (twice where it does not fit a workgroup), y written once.  Two forms:
//
//   one launch   a workgroup holds whole groups of one sample in its registers, all positions of them: mean, then the squared
//                deviations from it, then the result, with no second look at memory.  Taken where that fits: some groups of a
//                sample (norm_resident: their lanes have to be powers of two; norm_sample: any, or the whole sample).
//   two launches statistics of stretches of positions (each: mean and sum of squared deviations, put together pairwise, never as
//                a difference of large sums), then the result, whose workgroups first put their sample's stretches together.
//                x comes from the last-level cache the second time where it fits there (256 MB).
//
// Measured: 32 x 56x56 x 256 fp32 (206 MB) 45-47 us, 4.4 TB/s, where a copy of as much takes 40; 7x7 x 2048 f16 4.5 us on the GPU, little more than a
// launch; 7 x 27x31 x 360 bf16 to codes (groups of 12) in two launches 6.4 + 8.2 us, each a launch, one or two trips to memory and its arithmetic.
#include "op_common.h"

#include <algorithm>
#include <cmath>
#include <numeric>

namespace sc {
namespace {

constexpr int kThreads = 256;                // of a workgroup of the two-launch form
constexpr int kMaxStretches = 64;            // stretches of positions of a sample
constexpr int kParts = 1024;                 // statistics that a workgroup of the second launch takes in at a time

struct NormArgs {
    const void* x;
    const float* gamma;
    const float* beta;
    void* y;
    float* ys;
    float2* stats;                           // [N][G][stretches][parts] mean, sum of squared deviations
    int N, S, C, G, Cg;
    int seg, segs, parts;                    // channels of a workgroup of whole samples' parts, or of the statistics, segments of C, segments of one group (1: whole groups)
    int len, stretches;                      // positions of a stretch, stretches of a sample
    int rows;                                // positions of a workgroup of the second launch
    int once;                                // x passes the last-level cache by
    float eps;
    int64_t x_sample, x_row, y_sample, y_row, s_row;
};

// V parameters from channel c on (the first `have`; `otherwise` where there are none).
template <int V> __device__ __forceinline__ void load_params(float* out, const float* p, int c, int have, float otherwise)
{
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = otherwise;
    if (!p || have <= 0) return;
    if (have >= V) {
        __builtin_memcpy(out, p + c, 4 * V);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = p[c + min(i, have - 1)];
    }
}

// floor(i / d) for 0 <= i < 2^19, inv = 1.0f / d: the half keeps the product away from whole numbers by more than it is rounded.
__device__ __forceinline__ int small_div(int i, float inv) { return (int)(((float)i + 0.5f) * inv); }

// y of V neighbouring channels of one position; gam: gamma over the spread.
template <int ACT, int YT, int V>
__device__ __forceinline__ void finish(float* f, const float* mean, const float* gam, const float* bet, int have)
{
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i < have ? activate<ACT, YT>((f[i] - mean[i]) * gam[i] + bet[i]) : 0.0f;
}

// The sample and part of this workgroup, of `parts` a sample.  dies: those of a sample go to one die, one after another, so that the pieces
// of a line that they read and write meet in its cache (workgroups are dealt to the eight dies in turn).
__device__ __forceinline__ void place(int parts, int dies, int& n, int& part)
{
    const int of = dies ? blockIdx.x >> 3 : blockIdx.x, at = of / parts;
    n = dies ? at * 8 + (blockIdx.x & 7) : at;
    part = of - at * parts;
}

// ---------------------------------------------------------------------------------------------------------------------------
// One launch.  TPR lanes side by side cover the channels of a workgroup (16 bytes each, a power of two, LPG of them a group), the
// others of the T lanes the positions; U positions a lane.  A sum over a group is a sum over lanes of a wave by shuffles and one over
// the waves through LDS.
// ---------------------------------------------------------------------------------------------------------------------------
template <int XT, int YT, int ACT, int T, int U> __global__ __launch_bounds__(T, 4) void norm_resident_kernel(NormArgs a, int TPR, int LPG, int dies)
{
    constexpr int V = kVec<XT>, W = T / 64;
    __shared__ float red[2][W][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int n, part;
    place(a.C / (TPR * V), dies, n, part);
    const int c0 = part * TPR * V;
    if (n >= a.N) return;
    const int col = threadIdx.x & (TPR - 1), r0 = threadIdx.x / TPR, R = T / TPR, c = c0 + col * V;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + c;
    v4i raw[U];
    if (a.once) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = v4i{0, 0, 0, 0};
            if (r0 + u * R < a.S) raw[u] = load_raw_once<XT>(x + (r0 + u * R) * a.x_row);
        }
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = v4i{0, 0, 0, 0};
            if (r0 + u * R < a.S) raw[u] = load_raw<XT>(x + (r0 + u * R) * a.x_row);
        }
    }
    float gam[V], bet[V];
    load_params<V>(gam, a.gamma, c, V, 1.0f);
    load_params<V>(bet, a.beta, c, V, 0.0f);
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
    // (the values are widened again for each pass: kept wide, two-byte types would not fit the registers)
    auto forget = [&] {
#pragma unroll
        for (int u = 0; u < U; ++u) asm volatile("" : "+v"(raw[u]));
    };
    forget();
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
    forget();
    float means[V];
#pragma unroll
    for (int i = 0; i < V; ++i) means[i] = mean, gam[i] *= inv;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int pos = r0 + u * R;
        if (pos >= a.S) continue;            // (a position's lanes go on or leave together: the shuffles below stay inside it)
        float f[V];
        to_floats<XT>(raw[u], f);
        finish<ACT, YT, V>(f, means, gam, bet, V);
        Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + n * a.y_sample + pos * a.y_row + c;
        if constexpr (YT == SC_ELEM_E4M3) {
            constexpr int L = kQBlock / V;
            float amax = kAmaxFloor;
#pragma unroll
            for (int i = 0; i < V; ++i) amax = fmaxf(amax, fabsf(f[i]));
            amax = max_block<L>(amax);
            store_codes<V>(y, f, kCodeMax / amax);
            if (col % L == 0) a.ys[((int64_t)n * a.S + pos) * a.s_row + c / kQBlock] = amax / kCodeMax;
        } else {
            store_vec<YT, V>(y, f, V);
        }
        if constexpr (U > 4) __builtin_amdgcn_sched_barrier(0);      // (one position at a time: sixteen under way do not fit the registers)
    }
}

// ---------------------------------------------------------------------------------------------------------------------------
// One launch, groups of any size: a workgroup holds a whole sample or the groups of whole vectors of it (a.seg channels; codes: of whole
// blocks), lanes side by side V neighbouring channels each.  Sums of channels go
// through LDS and are put together by group (by_group), for the mean and then for the squared deviations from it.
// ---------------------------------------------------------------------------------------------------------------------------
// out[g] = the sum of value(g, row, channel of the group) over R rows and gc channels: by several waves each for a few groups, by one
// for some, by sixteen lanes each for many.
template <int T, class F> __device__ __forceinline__ void by_group(int groups, int gc, int R, float* out, float* red, F value)
{
    const float inv = 1.0f / (float)gc;
    auto part = [&](int g, int first, int step) {
        float s = 0.0f;
        for (int i = first; i < R * gc; i += step) {
            const int rr = small_div(i, inv);
            s += value(g, rr, i - rr * gc);
        }
        return s;
    };
    const int per = T / 64 / groups, wave = threadIdx.x >> 6;
    if (per > 1) {
        const int g = wave / per;
        if (g < groups) {
            const float s = sum64(part(g, threadIdx.x - g * per * 64, per * 64));
            if ((threadIdx.x & 63) == 0) red[wave] = s;
        }
        __syncthreads();
        if ((int)threadIdx.x < groups) {
            float all = 0.0f;
            for (int w = 0; w < per; ++w) all += red[threadIdx.x * per + w];
            out[threadIdx.x] = all;
        }
    } else if (groups * 16 < T) {
        for (int g = wave; g < groups; g += T / 64) {
            const float s = sum64(part(g, threadIdx.x & 63, 64));
            if ((threadIdx.x & 63) == 0) out[g] = s;
        }
    } else {
        for (int g = threadIdx.x >> 4; g < groups; g += T / 16) {
            const float s = sum16(part(g, threadIdx.x & 15, 16));
            if ((threadIdx.x & 15) == 0) out[g] = s;
        }
    }
    __syncthreads();
}

template <int XT, int YT, int ACT, int T, int U> __global__ __launch_bounds__(T, 4) void norm_sample_kernel(NormArgs a, int dies)
{
    constexpr int V = kVec<XT>, L = kQBlock / V;
    constexpr bool CODES = YT == SC_ELEM_E4M3;
    __shared__ float vals[T * V], red[T / 64];
    extern __shared__ float by[];                    // [2][G]
    int n, part;
    place(a.segs, dies, n, part);
    if (n >= a.N) return;
    const int c0 = part * a.seg, C = min(a.seg, a.C - c0), G = C / a.Cg;      // its channels: C from c0 on
    const int tpr = CODES ? (C + kQBlock - 1) / kQBlock * L : (C + V - 1) / V, R = small_div(T, 1.0f / (float)tpr);
    const int r = small_div(threadIdx.x, 1.0f / (float)tpr), v = threadIdx.x - r * tpr, c = v * V;
    const int have = min(V, C - c), rows = r < R ? a.S : 0;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + c0 + c;
    v4i raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        raw[u] = v4i{0, 0, 0, 0};
        if (r + u * R < rows && have > 0) raw[u] = have == V ? load_raw<XT>(x + (r + u * R) * a.x_row) : load_raw_part<XT>(x + (r + u * R) * a.x_row, have);
    }
    float gam[V], bet[V];
    load_params<V>(gam, a.gamma, c0 + c, have, 1.0f);
    load_params<V>(bet, a.beta, c0 + c, have, 0.0f);
    const float cnt = (float)a.S * (float)a.Cg;
    const int first = min(c, C - 1) / a.Cg, ends = (first + 1) * a.Cg - c;   // the group of a lane's first channel, its channels to come
    auto each = [&](const float* t, auto take) {     // take(i, t of the group of channel c + i)
        int g = first, left = ends;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            take(i, t[min(g, G - 1)]);
            if (--left == 0) ++g, left = a.Cg;
        }
    };
    auto forget = [&] {                              // (see norm_resident_kernel)
#pragma unroll
        for (int u = 0; u < U; ++u) asm volatile("" : "+v"(raw[u]));
    };
    float sum[V] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float f[V];
        to_floats<XT>(raw[u], f);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += f[i];
    }
    auto together = [&](float* out) {
#pragma unroll
        for (int i = 0; i < V; ++i) vals[threadIdx.x * V + i] = sum[i];
        __syncthreads();
        by_group<T>(G, a.Cg, R, out, red, [&](int g, int rr, int cc) { return vals[rr * tpr * V + g * a.Cg + cc]; });
    };
    together(by);
    forget();
    float mean[V];
    each(by, [&](int i, float t) { mean[i] = t / cnt, sum[i] = 0.0f; });
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (r + u * R < rows) {
            float f[V];
            to_floats<XT>(raw[u], f);
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += (f[i] - mean[i]) * (f[i] - mean[i]);
        }
    together(by + G);
    forget();
    each(by + G, [&](int i, float t) { gam[i] *= 1.0f / sqrtf(t / cnt + a.eps); });
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int pos = r + u * R;
        if (pos >= rows) continue;                   // (the lanes of a position go on or leave together)
        float f[V];
        to_floats<XT>(raw[u], f);
        finish<ACT, YT, V>(f, mean, gam, bet, have);
        Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + n * a.y_sample + pos * a.y_row + c0 + c;
        if constexpr (CODES) {
            float amax = kAmaxFloor;
#pragma unroll
            for (int i = 0; i < V; ++i) amax = fmaxf(amax, fabsf(f[i]));
            amax = max_block<L>(amax);
            if (c < ((C + 15) & ~15)) store_codes<V>(y, f, kCodeMax / amax);
            if (v % L == 0) a.ys[((int64_t)n * a.S + pos) * a.s_row + (c0 + c) / kQBlock] = amax / kCodeMax;
        } else {
            store_vec<YT, V>(y, f, have);
        }
        if constexpr (U > 4) __builtin_amdgcn_sched_barrier(0);
    }
}

// ---------------------------------------------------------------------------------------------------------------------------
// Two launches, the first: one workgroup per (sample, stretch of positions, segment of channels).  A lane keeps V neighbouring
// channels and takes U positions at a time: their mean, their squared deviations from it, and both joined to what it has.
// ---------------------------------------------------------------------------------------------------------------------------
template <int XT> __global__ __launch_bounds__(kThreads) void norm_stats_kernel(NormArgs a)
{
    constexpr int V = kVec<XT>, U = 8;
    __shared__ float ms[kThreads * V], qs[kThreads * V], ns[kThreads], red[kThreads / 64], by[2 * kThreads * V];
    const int n = blockIdx.x, st = blockIdx.y, sg = blockIdx.z;
    // (a.parts > 1: a segment is a part of one group; else whole groups)
    const int g0 = a.parts > 1 ? sg / a.parts : sg * (a.seg / a.Cg), part = a.parts > 1 ? sg % a.parts : 0;
    const int c0 = a.parts > 1 ? g0 * a.Cg + part * a.seg : sg * a.seg;
    const int cn = a.parts > 1 ? min(a.seg, a.Cg - part * a.seg) : min(a.seg, a.C - c0);
    const int tpr = (cn + V - 1) / V, R = small_div(kThreads, 1.0f / (float)tpr);
    const int r = small_div(threadIdx.x, 1.0f / (float)tpr), v = threadIdx.x - r * tpr;
    const int p0 = st * a.len, pn = min(a.len, a.S - p0);
    const int have = min(V, cn - v * V);
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + p0 * a.x_row + c0 + v * V;
    float mean[V] = {}, m2[V] = {}, cnt = 0.0f;
    // (A batch is U positions, the last one as many as there are; the loads of a batch are under way while the one before is added up.)
    auto load = [&](v4i* raw, int p) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = v4i{0, 0, 0, 0};
            if (p + u * R < pn) raw[u] = have == V ? load_raw<XT>(x + (p + u * R) * a.x_row) : load_raw_part<XT>(x + (p + u * R) * a.x_row, have);
        }
    };
    if (r < R) {
        v4i raw[U];
        load(raw, r);
        for (int p = r; p < pn; p += U * R) {
            v4i now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) now[u] = raw[u];
            if (p + U * R < pn) load(raw, p + U * R);
            const int valid = min(U, (pn - p + R - 1) / R);
            const float n2 = (float)valid, share = n2 / (cnt + n2), each = 1.0f / n2;
            float sum[V] = {}, sq[V] = {};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[V];
                to_floats<XT>(now[u], f);
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] += f[i];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] *= each;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float f[V];
                to_floats<XT>(now[u], f);
                if (u < valid)
#pragma unroll
                    for (int i = 0; i < V; ++i) sq[i] += (f[i] - sum[i]) * (f[i] - sum[i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = sum[i] - mean[i];
                mean[i] += d * share;
                m2[i] += sq[i] + d * d * cnt * share;
            }
            cnt += n2;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ms[threadIdx.x * V + i] = mean[i];
        qs[threadIdx.x * V + i] = m2[i];
    }
    ns[threadIdx.x] = r < R ? cnt : 0.0f;
    __syncthreads();
    // The groups: the mean of the means, then the deviations around it.
    const int groups = a.parts > 1 ? 1 : cn / a.Cg, gc = a.parts > 1 ? cn : a.Cg;
    const float total = (float)pn * (float)gc;
    by_group<kThreads>(groups, gc, R, by, red, [&](int g, int rr, int cc) {
        cc += g * gc;
        return ns[rr * tpr + cc / V] * ms[rr * tpr * V + cc];
    });
    for (int g = threadIdx.x; g < groups; g += kThreads) by[g] /= total;
    __syncthreads();
    by_group<kThreads>(groups, gc, R, by + groups, red, [&](int g, int rr, int cc) {
        cc += g * gc;
        const float d = ms[rr * tpr * V + cc] - by[g];
        return qs[rr * tpr * V + cc] + ns[rr * tpr + cc / V] * d * d;
    });
    for (int g = threadIdx.x; g < groups; g += kThreads)
        a.stats[(((int64_t)n * a.G + g0 + g) * a.stretches + st) * a.parts + part] = make_float2(by[g], by[groups + g]);
}

// The second: one workgroup per (sample, a.rows positions, up to kThreads * V channels).  Codes: a row's lanes are padded to whole
// blocks of 128 channels, so that a block's lanes are neighbours in one wave.
template <int XT, int YT, int ACT> __global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a, int wide)
{
    constexpr int V = kVec<XT>, U = 4, L = kQBlock / V;
    constexpr bool CODES = YT == SC_ELEM_E4M3;
    extern __shared__ float2 gs[];           // mean, 1 / spread of the groups of this workgroup
    const int n = blockIdx.x, ch = blockIdx.y, sg = blockIdx.z;
    const int c0 = sg * wide, cn = min(wide, a.C - c0);
    const int tpr = CODES ? (cn + kQBlock - 1) / kQBlock * L : (cn + V - 1) / V;
    const int R = small_div(kThreads, 1.0f / (float)tpr), r = small_div(threadIdx.x, 1.0f / (float)tpr), v = threadIdx.x - r * tpr;
    const int have = min(V, cn - v * V), c = c0 + v * V;
    const int p0 = ch * a.rows, p1 = r < R ? min(a.S, p0 + a.rows) : 0;
    const Elem<XT>* x = static_cast<const Elem<XT>*>(a.x) + n * a.x_sample + c;
    Elem<YT>* y = static_cast<Elem<YT>*>(a.y) + n * a.y_sample + c;
    v4i raw[U];
    auto load = [&](int p) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = v4i{0, 0, 0, 0};
            if (p + u * R < p1 && have > 0) raw[u] = have == V ? load_raw<XT>(x + (p + u * R) * a.x_row) : load_raw_part<XT>(x + (p + u * R) * a.x_row, have);
        }
    };
    // (what does not depend on the statistics is on its way while they are put together)
    load(p0 + r);
    float gam[V], bet[V];
    load_params<V>(gam, a.gamma, c, have, 1.0f);
    load_params<V>(bet, a.beta, c, have, 0.0f);
    const int g0 = c0 / a.Cg, groups = (c0 + cn - 1) / a.Cg - g0 + 1;
    // The stretches of as many groups as fit, all of them asked for at once (they come from the other dies' caches, 1-2 us away),
    // then sixteen lanes a group.
    __shared__ float2 parts_[kParts];
    const int sub = threadIdx.x >> 4, sl = threadIdx.x & 15, per = a.stretches * a.parts, at_once = kParts / per;
    const float total = (float)a.S * (float)a.Cg;
    for (int gb = 0; gb < groups; gb += at_once) {
        const int gn = min(at_once, groups - gb);
        const float2* st = a.stats + ((int64_t)n * a.G + g0 + gb) * per;
        float2 got[kParts / kThreads];
#pragma unroll
        for (int k = 0; k < kParts / kThreads; ++k)
            if ((int)threadIdx.x + k * kThreads < gn * per) got[k] = st[threadIdx.x + k * kThreads];
        if (gb) __syncthreads();
#pragma unroll
        for (int k = 0; k < kParts / kThreads; ++k)
            if ((int)threadIdx.x + k * kThreads < gn * per) parts_[threadIdx.x + k * kThreads] = got[k];
        __syncthreads();
        for (int g = sub; g < gn; g += kThreads / 16) {
            auto count = [&](int i) {
                const int st_ = a.parts > 1 ? i / a.parts : i, part = i - st_ * a.parts;
                return (float)min(a.len, a.S - st_ * a.len) * (float)(a.parts > 1 ? min(a.seg, a.Cg - part * a.seg) : a.Cg);
            };
            float mean = 0.0f, m2 = 0.0f;
            for (int i = sl; i < per; i += 16) mean += count(i) * parts_[g * per + i].x;
            mean = sum16(mean) / total;
            for (int i = sl; i < per; i += 16) {
                const float2 q = parts_[g * per + i];
                m2 += q.y + count(i) * (q.x - mean) * (q.x - mean);
            }
            m2 = sum16(m2);
            if (sl == 0) gs[gb + g] = make_float2(mean, 1.0f / sqrtf(m2 / total + a.eps));
        }
    }
    __syncthreads();
    float mean[V];
    const int first = min(c, a.C - 1) / a.Cg;
    int g = first, left = (first + 1) * a.Cg - c;            // (the group of a channel, and how many of its channels are to come)
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = gs[min(g - g0, groups - 1)];
        mean[i] = s.x, gam[i] *= s.y;
        if (--left == 0) ++g, left = a.Cg;
    }
    for (int p = p0 + r; p < p1; p += U * R) {
        v4i now[U];
#pragma unroll
        for (int u = 0; u < U; ++u) now[u] = raw[u];
        if (p + U * R < p1) load(p + U * R);
        float f[U][V], amax[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            to_floats<XT>(now[u], f[u]);
            finish<ACT, YT, V>(f[u], mean, gam, bet, have);
            if constexpr (CODES) {
                amax[u] = kAmaxFloor;
#pragma unroll
                for (int i = 0; i < V; ++i) amax[u] = fmaxf(amax[u], fabsf(f[u][i]));
                amax[u] = max_block<L>(amax[u]);         // (a block's lanes have the same position: all of it counts or none)
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int pos = p + u * R;
            if (pos >= p1) break;
            if constexpr (CODES) {
                if (c < ((a.C + 15) & ~15)) store_codes<V>(y + pos * a.y_row, f[u], kCodeMax / amax[u]);
                if (v % L == 0) a.ys[((int64_t)n * a.S + pos) * a.s_row + c / kQBlock] = amax[u] / kCodeMax;
            } else {
                store_vec<YT, V>(y + pos * a.y_row, f[u], have);
            }
        }
    }
}

constexpr int kNumUnits = 256;                // compute units
constexpr int64_t kMaxThreads = (int64_t)1 << 32;   // of a launch: below this

bool pow2(int v) { return v > 0 && (v & (v - 1)) == 0; }

struct NormShape {
    int T, U;                                // one launch (T = 0: two)
    int dies, TPR, LPG;                      // ... of lanes in powers of two (TPR = 0: of whole samples or parts of them: seg, segs)
    int seg, segs, parts, len, stretches;    // the statistics
    int wide, wides, rows, chunks;           // the result
    size_t bytes;
};

// What a form takes, in microseconds: one launch 4.5 (norm_sample 5.5), two 11.5; then the larger of what memory takes at 4.5 TB/s and, for one
// launch of `parts` workgroups a sample, what the fullest of 256 compute units takes at 5500 values a microsecond (three passes of 17 vector
// instructions in all for each value).  `reads`: how often a line comes from memory where the parts of a sample are on several dies; on one die
// (`dies`) it comes once, but there are 32 compute units and an eighth of the bandwidth for each sample.
// Measured for estimated: 7 x 837 x 360 to codes 13.9 for 13.8, 4 x 3000 x 416 17.0 for 18.2,
// 1 x 3136 x 64 (8 groups, f16) 8.6 for 9.1 (four workgroups on several dies 11.3), 29 x 1883 x 64 (32 groups, bf16) 12.9 for 8.6 (15.3).
double norm_time(const sc_group_norm_t* d, double base, double parts, double values, double reads, int* dies)
{
    const double total = (double)d->N * d->S * d->C, x = elem_bytes(d->x_type), y = elem_bytes(d->y_type);
    const double spread = std::max(std::ceil(d->N * parts / kNumUnits) * values / 5500.0, total * (reads * x + y) / 4.5e6);
    const double held = std::max(std::ceil(std::ceil(d->N / 8.0) * parts / (kNumUnits / 8)) * values / 5500.0, total * (x + y) / (4.5e6 * std::min(d->N, 8) / 8));
    *dies = parts > 1.0 && held <= spread;
    return base + (*dies ? held : spread);
}

// One launch: groups of a power of two of 16-byte lanes, all positions of a workgroup's channels in 16 vectors a lane of 1024.  The
// channels of a workgroup make a whole line of 128 bytes, or a part of one (codes: whole blocks of 128 channels).
bool norm_resident(const sc_group_norm_t* d, NormShape* s, double* time)
{
    const int V = 16 / elem_bytes(d->x_type), Cg = d->C / d->G;
    const bool codes = d->y_type == SC_ELEM_E4M3;
    if (Cg % V || !pow2(Cg / V) || Cg / V > 64) return false;
    const int LPG = Cg / V, line = codes ? kQBlock / V : 8, least = codes ? line : 1;
    bool any = false;
    for (int TPR = LPG; TPR <= std::max(line, LPG) && d->C % (TPR * V) == 0; TPR *= 2) {
        const int64_t vectors = (int64_t)d->S * TPR;
        if (TPR < least || TPR % (codes ? line : 1) || vectors > 1024 * 16) continue;
        int dies;
        const double t = norm_time(d, 4.5, d->C / (TPR * V), (double)vectors * V, std::max(1.0, 8.0 / TPR), &dies);
        if (ceil_div(d->N, 8) * 8 * (d->C / (TPR * V)) * 1024 >= kMaxThreads || (any && t > *time)) continue;      // (level: the wider)
        any = true;
        *time = t;
        s->TPR = TPR;
        s->LPG = LPG;
        s->dies = dies;
        s->T = vectors <= 256 * 4 ? 256 : vectors <= 512 * 16 ? 512 : 1024;
        s->U = vectors <= s->T * 4 ? 4 : 16;
    }
    return any;
}

// One launch, a sample a workgroup, or a part of one: the fewest groups that fill vectors (codes: blocks), times a power of two.  In
// eight vectors a lane of 1024.  (64 x 49 x 1040, 16 groups, f16: whole samples 15.7 us, halves of them
// 12.7; 6 x 427 x 1152, 16 groups, fp32: two launches 17.7, a workgroup a group 11.7.)
bool norm_sample(const sc_group_norm_t* d, NormShape* s, double* time)
{
    const int V = 16 / elem_bytes(d->x_type), L = kQBlock / V;
    const bool codes = d->y_type == SC_ELEM_E4M3;
    bool any = false;
    for (int64_t part = std::lcm<int64_t>(d->C / d->G, codes ? kQBlock : V);; part *= 2) {
        part = std::min<int64_t>(part, d->C);
        const int64_t tpr = codes ? ceil_div(part, kQBlock) * L : ceil_div(part, V), segs = ceil_div(d->C, part), bytes = part * elem_bytes(d->x_type);
        if (tpr <= 1024 && part / (d->C / d->G) <= 2048 && ceil_div(d->N, 8) * 8 * segs * 1024 < kMaxThreads) {
            const int T = tpr <= 256 && 256 / tpr * 4 >= d->S ? 256 : 1024, U = T / tpr * 4 >= d->S ? 4 : 8;
            // (parts that share lines read them twice)
            int dies;
            const double t = norm_time(d, 5.5, (double)segs, (double)d->S * part, segs == 1 || bytes % 128 == 0 ? 1.0 : 1.0 + 128.0 / bytes, &dies);
            if (T / tpr * U >= d->S && (!any || t <= *time)) {
                any = true;
                *time = t;
                s->T = T;
                s->U = U;
                s->dies = dies;
                s->seg = (int)part;
                s->segs = (int)segs;
            }
        }
        if (part == d->C) return any;
    }
}

NormShape norm_shape(const sc_group_norm_t* d)
{
    if (d->N == 0 || d->S == 0) return {};
    NormShape one{}, resident{}, sample{};
    double best = norm_time(d, 11.5, 0.0, 0.0, 2.0, &one.dies), time = 0.0;
    if (norm_resident(d, &resident, &time) && time < best) one = resident, best = time;
    if (norm_sample(d, &sample, &time) && time < best) one = sample;
    if (one.T) return one;
    NormShape s{};
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
    // Four workgroups a compute unit for the first launch, eight for the second, no stretch under eight vectors a lane, no fewer than four a lane in the
    // second (7 x 837 x 360 to codes: 13.9 us; five vectors a lane in the first 14.3, twelve 14.7; two in the second 14.4, eight 15.5).
    const int R = std::max<int>(1, kThreads / (int)ceil_div(std::min(s.seg, d->C), V));
    const int64_t want = std::max<int64_t>(1, 1024 / ((int64_t)d->N * s.segs));
    s.stretches = (int)std::min<int64_t>({want, kMaxStretches, kParts / s.parts, ceil_div(d->S, 8 * R)});
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

// Whether x and y do not stay in the last-level cache side by side: x passes it by then.
// (32 x 56x56 x 256 fp32, 206 MB: 47 us with the hint and 52 without; 39 MB of a quantiser's: 11.0 with and 10.4 without)
bool past_cache(const sc_group_norm_t* d) { return (int64_t)d->N * d->S * d->C * (elem_bytes(d->x_type) + elem_bytes(d->y_type)) > (int64_t)128 << 20; }

sc_status_t check_norm(const sc_group_norm_t* d)
{
    if (!d) return SC_ERR_NULL;
    if (d->N < 0 || d->S < 0 || d->C <= 0 || d->G <= 0 || d->C % d->G) return SC_ERR_SHAPE;
    if (!is_wide(d->x_type) || (d->y_type != d->x_type && d->y_type != SC_ELEM_E4M3)) return SC_ERR_UNSUPPORTED;
    if (d->act < SC_ACT_NONE || d->act > SC_ACT_SILU || !(d->eps >= 0.0f) || d->eps > 3e38f) return SC_ERR_UNSUPPORTED;
    if ((int64_t)d->S * d->C >= (int64_t)1 << 31 || (int64_t)d->N * d->S >= (int64_t)1 << 31) return SC_ERR_RANGE;
    if (d->S > 1 << 30) return SC_ERR_RANGE;                 // (a workgroup looks up to its own number of positions beyond its last one, in 32 bits)
    if (d->C / d->G >= 1 << 20) return SC_ERR_RANGE;         // (the parts of a group: kParts of 1024 channels or more)
    if (d->x_sample < 0 || d->x_row < 0) return SC_ERR_SHAPE;
    if (d->y_row < d->C) return SC_ERR_SHAPE;
    if (d->N > 1 && d->S > 0 && d->y_sample < (__int128)(d->S - 1) * d->y_row + d->C) return SC_ERR_SHAPE;      // (the product may pass 64 bits)
    if (d->y_type == SC_ELEM_E4M3) {
        if (d->scale_row < ceil_div(d->C, kQBlock)) return SC_ERR_SHAPE;
        if (d->y_row % 16 || d->y_sample % 16) return SC_ERR_UNSUPPORTED;
    }
    return SC_OK;
}

template <int XT, int YT, int ACT> sc_status_t launch_norm(const sc_group_norm_t* d, const NormShape& s, const NormArgs& a, hipStream_t stream)
{
    const int64_t samples = s.dies ? ceil_div(d->N, 8) * 8 : (int64_t)d->N;
    if (s.T && !s.TPR) {
        const size_t lds = (size_t)(s.seg / a.Cg) * 2 * sizeof(float);
        const dim3 grid((unsigned)(samples * s.segs));
        if (s.T == 256) norm_sample_kernel<XT, YT, ACT, 256, 4><<<grid, 256, lds, stream>>>(a, s.dies);
        else if (s.U == 4) norm_sample_kernel<XT, YT, ACT, 1024, 4><<<grid, 1024, lds, stream>>>(a, s.dies);
        else norm_sample_kernel<XT, YT, ACT, 1024, 8><<<grid, 1024, lds, stream>>>(a, s.dies);
        return launched();
    }
    if (s.T) {
        const dim3 grid((unsigned)(samples * (d->C / (s.TPR * kVec<XT>))));
        if (s.T == 256) norm_resident_kernel<XT, YT, ACT, 256, 4><<<grid, 256, 0, stream>>>(a, s.TPR, s.LPG, s.dies);
        else if (s.U == 4) norm_resident_kernel<XT, YT, ACT, 512, 4><<<grid, 512, 0, stream>>>(a, s.TPR, s.LPG, s.dies);
        else if (s.T == 512) norm_resident_kernel<XT, YT, ACT, 512, 16><<<grid, 512, 0, stream>>>(a, s.TPR, s.LPG, s.dies);
        else norm_resident_kernel<XT, YT, ACT, 1024, 16><<<grid, 1024, 0, stream>>>(a, s.TPR, s.LPG, s.dies);
        return launched();
    }
    const int64_t first = (int64_t)d->N * s.segs * s.stretches, second = (int64_t)d->N * s.wides * s.chunks;
    if (std::max(first, second) * kThreads >= (int64_t)1 << 32 || std::max({s.segs, s.wides, s.chunks}) > 65535) return SC_ERR_RANGE;
    norm_stats_kernel<XT><<<dim3((unsigned)d->N, (unsigned)s.stretches, (unsigned)s.segs), kThreads, 0, stream>>>(a);
    if (launched() != SC_OK) return SC_ERR_HIP;
    const size_t lds = (size_t)std::min<int64_t>(d->G, ceil_div(s.wide, a.Cg) + 1) * sizeof(float2);
    norm_apply_kernel<XT, YT, ACT><<<dim3((unsigned)d->N, (unsigned)s.chunks, (unsigned)s.wides), kThreads, lds, stream>>>(a, s.wide);
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

extern "C" sc_status_t sparse_conv_group_norm_launch(const sc_group_norm_t* d, sc_launch_t* launch)
{
    if (!launch) return SC_ERR_NULL;
    const sc_status_t st = check_norm(d);
    if (st != SC_OK) return st;
    *launch = sc_launch_t{};
    if (d->N == 0 || d->S == 0) return SC_OK;
    const NormShape s = norm_shape(d);
    launch->form = !s.T ? SC_FORM_NORM_TWO : s.TPR ? SC_FORM_NORM_LANES : SC_FORM_NORM_SAMPLE;
    launch->lanes = s.T;
    launch->held = s.U;
    launch->one_die = s.T ? s.dies : 0;
    launch->past_cache = s.T && s.TPR && past_cache(d);
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
    a.once = past_cache(d);
    a.x_sample = d->x_sample; a.x_row = d->x_row; a.y_sample = d->y_sample; a.y_row = d->y_row; a.s_row = d->scale_row;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (d->x_type) {
        case SC_ELEM_F32: return launch_norm<SC_ELEM_F32>(d, shape, a, s);
        case SC_ELEM_F16: return launch_norm<SC_ELEM_F16>(d, shape, a, s);
        default: return launch_norm<SC_ELEM_BF16>(d, shape, a, s);
    }
}
