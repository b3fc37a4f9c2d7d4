// The router of a layer of experts (sparse_conv_route_experts, _backward).
//
// L lanes hold the E logits of a token, V each, and take the largest out `top` times: the largest of a lane's, then four (sixteen lanes) or six
// exchanges, and the lane that holds it drops it.  What is compared is one number that has the expert in its low bits, so that
// equal logits go by rising number of themselves: 32 bits for 16-bit logits, 64 for 32-bit ones.  With a bias the sums are taken
// in 64 bits, since scores in 32 bits lie next to one another too often for a choice that has to be repeatable; the expert takes the last twelve of
// them.  What bounds it is the vector unit: 16384 x 128 logits of 16 bits, top 8 (4096 waves), 11.1 us with comparisons of floats and numbers
// and the library's exponential and division, 10.7 without, 10.2 with sorted keys (see choose; calls back to back, the kernel alone takes 10.1).
#include "op_common.h"

#include <cmath>

namespace sc {
namespace {

struct RouteArgs {
    const void* x;
    const float* bias;
    const int32_t* ids_in;
    const float* dweights;
    int32_t* ids;
    float* weights;
    void* dx;
    int T, E, top, score, normalize;
    float factor;
    int64_t x_row, dx_row;
};

template <int N> __device__ __forceinline__ uint32_t ror_bits(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N, 0xf, 0xf, false); }
template <int N> __device__ __forceinline__ uint64_t ror_bits(uint64_t v)
{
    return (uint64_t)ror_bits<N>((uint32_t)(v >> 32)) << 32 | ror_bits<N>((uint32_t)v);
}
template <int N, class T> __device__ __forceinline__ T ror_any(T v)
{
    if constexpr (sizeof(T) == 8) return __builtin_bit_cast(T, ror_bits<N>(__builtin_bit_cast(uint64_t, v)));
    else return __builtin_bit_cast(T, ror_bits<N>(__builtin_bit_cast(uint32_t, v)));
}
// Of two copies of a value: the rows of sixteen lanes (32: the halves) that are even in both places, and those that are odd.
template <int N> __device__ __forceinline__ void swap_bits(uint32_t& a, uint32_t& b)
{
    const auto r = N == 16 ? __builtin_amdgcn_permlane16_swap(a, b, false, false) : __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
template <int N, class T> __device__ __forceinline__ void swap_any(T& a, T& b)
{
    uint32_t p[sizeof(T) / 4], q[sizeof(T) / 4];
    __builtin_memcpy(p, &a, sizeof(T));
    __builtin_memcpy(q, &b, sizeof(T));
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 4; ++i) swap_bits<N>(p[i], q[i]);
    __builtin_memcpy(&a, p, sizeof(T));
    __builtin_memcpy(&b, q, sizeof(T));
}
// f over the L lanes of a token (16 or 64), the same in all of them; all lanes of the wave come here.
template <int L, class T, class F> __device__ __forceinline__ T over_lanes(T v, F f)
{
    v = f(v, ror_any<8>(v));
    v = f(v, ror_any<4>(v));
    v = f(v, ror_any<2>(v));
    v = f(v, ror_any<1>(v));
    if constexpr (L == 64) {
        T other = v;
        swap_any<16>(v, other);
        v = f(v, other);
        other = v;
        swap_any<32>(v, other);
        v = f(v, other);
    }
    return v;
}
template <int L> __device__ __forceinline__ float lanes_sum(float v) { return over_lanes<L>(v, [](float a, float b) { return a + b; }); }
template <int L> __device__ __forceinline__ float lanes_max(float v) { return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); }); }

// Number e of a lane's value v: sixteen bytes in a row, then the next lane's.
template <int XT, int L> __device__ __forceinline__ int expert_of(int v, int lane) { return (v / kVec<XT> * L + lane) * kVec<XT> + v % kVec<XT>; }

// A lane's logits as floats, -inf where there is none or a NaN.
template <int XT, int L, int V> __device__ __forceinline__ void load_logits(const Elem<XT>* row, int E, int lane, float (&x)[V])
{
    constexpr int N = kVec<XT>;
#pragma unroll
    for (int c = 0; c < V / N; ++c) {
        const int e = (c * L + lane) * N;
        to_floats<XT>(e + N <= E ? load_raw<XT>(row + e) : load_raw_part<XT>(row + e, E - e), x + c * N);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e + i >= E || x[c * N + i] != x[c * N + i]) x[c * N + i] = -INFINITY;
    }
}

// What is compared without a bias: a number that rises with the logit and, for equal ones, falls with the expert's number; 0: none.
template <int XT> struct Key {
    using T = uint32_t;
    static __device__ __forceinline__ T make(float x, int e)
    {
        const uint16_t u = __builtin_bit_cast(uint16_t, (Elem<XT>)(x + 0.0f));       // (-0 is 0)
        return x > -INFINITY ? (uint32_t)(uint16_t)(u & 0x8000 ? ~u : u | 0x8000) << 16 | (0xffffu - (uint32_t)e) : 0;
    }
    static __device__ __forceinline__ int expert(T k) { return (int)(0xffffu - (k & 0xffffu)); }
    static __device__ __forceinline__ float logit(T k)
    {
        const uint16_t o = (uint16_t)(k >> 16);
        return (float)__builtin_bit_cast(Elem<XT>, (uint16_t)(o & 0x8000 ? o & 0x7fff : ~o));
    }
};
template <> struct Key<SC_ELEM_F32> {
    using T = uint64_t;
    static __device__ __forceinline__ T make(float x, int e)
    {
        const uint32_t u = __builtin_bit_cast(uint32_t, x + 0.0f);
        return x > -INFINITY ? (uint64_t)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | (0xffffffffu - (uint32_t)e) : 0;
    }
    static __device__ __forceinline__ int expert(T k) { return (int)(0xffffffffu - (uint32_t)k); }
    static __device__ __forceinline__ float logit(T k)
    {
        const uint32_t o = (uint32_t)(k >> 32);
        return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o);
    }
};

// The `top` largest keys of a token's L lanes, one after the other; a lane gets that of its own number, or 0 where there is none.  With eight keys a
// lane and six choices or more a lane's keys are sorted first (Batcher's merges of odd and even places), so that a choice compares the lanes' largest and one
// lane moves up; else all are compared for every choice (16384 tokens, us a call, compared and sorted: 128 experts, bias, top 8 10.7 and 10.2, top 4 8.1 and 8.3; 64, top 2 4.3 and
// 4.8; 256, sixteen keys a lane, top 8 12.4 and 16.9; 28936 x 56, bias, top 16 24.3 and 19.8; 15376 x 512, top 16 21 and 18, bias 51 and 42).
template <int L, class T, int V> __device__ __forceinline__ T choose(T (&key)[V], int top, int lane)
{
    T slot = 0;
    auto largest = [](T p, T q) { return p > q ? p : q; };
    if (V == 8 && top >= 6) {
#pragma unroll
        for (int p = 1; p < V; p *= 2)
#pragma unroll
            for (int k = p; k > 0; k /= 2)
#pragma unroll
                for (int j = k % p; j + k < V; j += 2 * k)
#pragma unroll
                    for (int i = j; i < j + k; ++i)
                        if (i + k < V && i / (2 * p) == (i + k) / (2 * p)) {
                            const T a = key[i], b = key[i + k];
                            key[i] = a > b ? a : b;
                            key[i + k] = a > b ? b : a;
                        }
        for (int j = 0; j < top; ++j) {
            const T best = over_lanes<L>(key[0], largest);
            const bool mine = key[0] == best;
#pragma unroll
            for (int v = 0; v < V - 1; ++v) key[v] = mine ? key[v + 1] : key[v];
            key[V - 1] = mine ? 0 : key[V - 1];
            if (lane == j) slot = best;
        }
    } else {
        for (int j = 0; j < top; ++j) {
            T best = key[0];
#pragma unroll
            for (int v = 1; v < V; ++v) best = largest(key[v], best);
            best = over_lanes<L>(best, largest);
#pragma unroll
            for (int v = 0; v < V; ++v) key[v] = key[v] == best ? 0 : key[v];
            if (lane == j) slot = best;
        }
    }
    return slot;
}

// exp of x <= 0 and the reciprocal of 1 and more in 64 bits, off by some 2^-51: x log2(e) = n + r with |r| <= 1/2, where r takes the product unrounded and the constant's
// lower half (from the rounded product it would be off by |x| 2^-53); the series of exp(r ln 2) up to the twelfth power, whose rest is 2e-16; 0 below e^-745, what 64 bits
// hold.  The hardware's reciprocal with two steps of Newton's.
__device__ __forceinline__ double exp64(double x)
{
    constexpr double kLog2e = 0x1.71547652b82fep+0, kLog2eLow = 0x1.777d0ffda0d24p-56;
    x = fmax(x, -746.0);
    const double n = rint(x * kLog2e), r = fma(x, kLog2eLow, fma(x, kLog2e, -n)) * 0x1.62e42fefa39efp-1;
    double p = 1.0 / 479001600.0;
    constexpr double k[] = {1.0 / 39916800.0, 1.0 / 3628800.0, 1.0 / 362880.0, 1.0 / 40320.0, 1.0 / 5040.0, 1.0 / 720.0, 1.0 / 120.0, 1.0 / 24.0, 1.0 / 6.0, 0.5, 1.0, 1.0};
#pragma unroll
    for (double c : k) p = fma(p, r, c);
    return ldexp(p, (int)n);
}
__device__ __forceinline__ double reciprocal64(double d)
{
    double r = __builtin_amdgcn_rcp(d);
    r = fma(fma(-d, r, 1.0), r, r);
    return fma(fma(-d, r, 1.0), r, r);
}

// A live slot's share of its token's score, a slot a lane.  Sigmoids are taken relative to the largest, exp(min(x, 0) - that of the
// largest) / (1 + exp(-|x|)), so that no sum of them is zero.  In 64 bits: one value a lane costs nothing beside the rest, and the weights are off by
// their rounding alone (in 32 bits 7.6e-8 of them).
template <int L> __device__ __forceinline__ float slot_share(float x, bool live, int score)
{
    const float lo = score == SC_SCORE_SIGMOID ? fminf(x, 0.0f) : x;
    const float top = lanes_max<L>(live ? lo : -INFINITY);
    double u;
    if (score == SC_SCORE_SIGMOID) u = exp64((double)lo - (double)top) * reciprocal64(1.0 + exp64(-fabs((double)x)));
    else u = exp((double)lo - (double)top);  // (a NaN where the largest is infinite)
    u = live ? u : 0.0;
    const double sum = over_lanes<L>(u, [](double p, double q) { return p + q; });
    return live ? (float)(u * reciprocal64(sum)) : 0.0f;
}
__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

template <int L, int V> __device__ __forceinline__ void row_softmax(const float (&x)[V], float& top, float& sum)
{
    top = x[0];
#pragma unroll
    for (int v = 1; v < V; ++v) top = fmaxf(top, x[v]);
    top = lanes_max<L>(top);
    sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) sum += x[v] > -INFINITY ? expf(x[v] - top) : 0.0f;
    sum = lanes_sum<L>(sum);
}

template <int XT, bool BIAS, int L, int V> __global__ __launch_bounds__(256) void route_pick_kernel(RouteArgs a)
{
    const int lane = threadIdx.x & (L - 1);
    const int t = blockIdx.x * (256 / L) + threadIdx.x / L, token = min(t, a.T - 1);       // (lanes without a token follow the last one's)
    float x[V];
    load_logits<XT, L, V>(static_cast<const Elem<XT>*>(a.x) + token * a.x_row, a.E, lane, x);
    int id = -1;
    float mine = 0.0f;                       // slot `lane`: its expert and logit
    if constexpr (!BIAS) {
        using K = Key<XT>;
        typename K::T key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = K::make(x[v], expert_of<XT, L>(v, lane));
        const typename K::T slot = choose<L>(key, a.top, lane);
        if (slot) id = K::expert(slot), mine = K::logit(slot);
    } else {
        double c[V];
        bool finite = true;                  // (a softmax of an infinite logit is a NaN for all)
        if (a.score == SC_SCORE_SOFTMAX) {
            float top = x[0];
#pragma unroll
            for (int v = 1; v < V; ++v) top = fmaxf(top, x[v]);
            top = lanes_max<L>(top);
            finite = top < INFINITY;
            double sum = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                c[v] = x[v] > -INFINITY ? exp64((double)x[v] - (double)top) : 0.0;
                sum += c[v];
            }
            sum = over_lanes<L>(sum, [](double p, double q) { return p + q; });
            const double inv = 1.0 / sum;
#pragma unroll
            for (int v = 0; v < V; ++v) c[v] *= inv;
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const double e = exp64(-fabs((double)x[v])), r = reciprocal64(1.0 + e);
                c[v] = x[v] < 0.0f ? e * r : r;
            }
        }
        uint64_t key[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int e = expert_of<XT, L>(v, lane);
            const double sum = c[v] + (double)a.bias[min(e, a.E - 1)] + 0.0;
            const uint64_t u = __builtin_bit_cast(uint64_t, sum);
            key[v] = x[v] > -INFINITY && finite && sum > (double)-INFINITY ? ((u >> 63 ? ~u : u | 1ull << 63) & ~4095ull) | (uint64_t)(4095 - (e & 4095)) : 0;
        }
        const uint64_t slot = choose<L>(key, a.top, lane);
        if (slot) id = 4095 - (int)(slot & 4095);
        if (id >= 0) mine = (float)(static_cast<const Elem<XT>*>(a.x) + token * a.x_row)[id];
    }
    const bool live = id >= 0;
    float w;
    if (a.normalize) w = slot_share<L>(mine, live, a.score);
    else if (a.score == SC_SCORE_SIGMOID) w = live ? sigmoid(mine) : 0.0f;
    else {
        float top, sum;
        row_softmax<L, V>(x, top, sum);
        w = live ? expf(mine - top) / sum : 0.0f;
    }
    if (t < a.T && lane < a.top) {
        a.ids[(int64_t)t * a.top + lane] = id;
        a.weights[(int64_t)t * a.top + lane] = w * a.factor;
    }
}

// dx = G - s D for a softmax that is not normalized (WHOLE: the row is read), else dx = G: G_e the sum over the slots with expert e of
//     softmax: g s;  normalized: p (g - sum g p);  sigmoid: g s (1 - s);  normalized: p (1 - s) (g - sum g p)
// with g = dweights * factor, p = s / sum s, D = the sum of all g s.
template <int XT, bool WHOLE, int L, int V> __global__ __launch_bounds__(256) void route_gradient_kernel(RouteArgs a)
{
    constexpr int N = kVec<XT>;
    const int lane = threadIdx.x & (L - 1), first = threadIdx.x & 63 & ~(L - 1);
    const int t = blockIdx.x * (256 / L) + threadIdx.x / L, token = min(t, a.T - 1);
    const Elem<XT>* row = static_cast<const Elem<XT>*>(a.x) + token * a.x_row;
    int id = lane < a.top ? a.ids_in[(int64_t)token * a.top + lane] : -1;
    float g = lane < a.top ? a.dweights[(int64_t)token * a.top + lane] * a.factor : 0.0f;
    float mine = (uint32_t)id < (uint32_t)a.E ? (float)row[id] : -INFINITY;
    const bool live = mine > -INFINITY;      // (and no NaN)
    if (!live) id = -1, g = 0.0f, mine = 0.0f;
    float x[V], top = 0.0f, sum = 1.0f, d, all = 0.0f;
    if constexpr (WHOLE) {
        load_logits<XT, L, V>(row, a.E, lane, x);
        row_softmax<L, V>(x, top, sum);
        d = live ? g * (expf(mine - top) / sum) : 0.0f;
        all = lanes_sum<L>(d);
    } else if (a.normalize) {
        const float p = slot_share<L>(mine, live, a.score);
        d = p * (g - lanes_sum<L>(g * p));
        if (a.score == SC_SCORE_SIGMOID) d *= sigmoid(-mine);
    } else {
        d = g * sigmoid(mine) * sigmoid(-mine);
    }
    float out[V] = {};
    for (int j = 0; j < a.top; ++j) {
        const int e = __shfl(id, first + j);
        const float add = __shfl(d, first + j);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (expert_of<XT, L>(v, lane) == e) out[v] += add;
    }
    if constexpr (WHOLE)
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (x[v] > -INFINITY) out[v] -= expf(x[v] - top) / sum * all;
    if (t >= a.T) return;
    Elem<XT>* dx = static_cast<Elem<XT>*>(a.dx) + (int64_t)t * a.dx_row;
#pragma unroll
    for (int c = 0; c < V / N; ++c) {
        const int e = (c * L + lane) * N;
        if (e < a.E) store_vec<XT, N>(dx + e, out + c * N, a.E - e);
    }
}

// Sixteen lanes a token up to 256 experts and 16 slots, the whole wave beyond.
template <int XT, bool BACK, bool B> sc_status_t launch_route(const RouteArgs& a, hipStream_t stream)
{
    const bool few = a.E <= 256 && a.top <= 16;
    const dim3 grid((unsigned)ceil_div(a.T, few ? 16 : 4));
    auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, stream>>>(a);
        return launched();
    };
    if constexpr (BACK) {
        if (few) return a.E <= 128 ? go(route_gradient_kernel<XT, B, 16, 8>) : go(route_gradient_kernel<XT, B, 16, 16>);
        return a.E <= 512 ? go(route_gradient_kernel<XT, B, 64, 8>) : a.E <= 1024 ? go(route_gradient_kernel<XT, B, 64, 16>) : go(route_gradient_kernel<XT, B, 64, 64>);
    } else {
        if (few) return a.E <= 128 ? go(route_pick_kernel<XT, B, 16, 8>) : go(route_pick_kernel<XT, B, 16, 16>);
        return a.E <= 512 ? go(route_pick_kernel<XT, B, 64, 8>) : a.E <= 1024 ? go(route_pick_kernel<XT, B, 64, 16>) : go(route_pick_kernel<XT, B, 64, 64>);
    }
}

sc_status_t check(const sc_route_experts_t* d, bool back)
{
    if (!d) return SC_ERR_NULL;
    if (d->T < 0 || d->E <= 0 || d->E > 4096 || d->top <= 0 || d->top > d->E || d->top > 64 || d->x_row < 0 || (back && d->dx_row < d->E)) return SC_ERR_SHAPE;
    if (!is_wide(d->x_type) || (d->score != SC_SCORE_SOFTMAX && d->score != SC_SCORE_SIGMOID) || (d->normalize != 0 && d->normalize != 1) || !std::isfinite(d->factor))
        return SC_ERR_UNSUPPORTED;
    if (d->T > 1 << 25) return SC_ERR_RANGE;                 // (64 threads a token fit a launch)
    return SC_OK;
}

RouteArgs args(const sc_route_experts_t* d, const void* x)
{
    RouteArgs a{};
    a.x = x;
    a.T = d->T; a.E = d->E; a.top = d->top; a.score = d->score; a.normalize = d->normalize; a.factor = d->factor;
    a.x_row = d->x_row; a.dx_row = d->dx_row;
    return a;
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" sc_status_t sparse_conv_route_experts(const sc_route_experts_t* d, const void* x, const float* bias, int32_t* ids, float* weights, void* stream)
{
    const sc_status_t st = check(d, false);
    if (st != SC_OK) return st;
    if (d->T == 0) return SC_OK;
    if (!x || !ids || !weights) return SC_ERR_NULL;
    if (!aligned(x, elem_bytes(d->x_type)) || !aligned(bias, 4) || !aligned(ids, 4) || !aligned(weights, 4)) return SC_ERR_UNSUPPORTED;
    RouteArgs a = args(d, x);
    a.bias = bias; a.ids = ids; a.weights = weights;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    switch (d->x_type) {
        case SC_ELEM_F32: return bias ? launch_route<SC_ELEM_F32, false, true>(a, s) : launch_route<SC_ELEM_F32, false, false>(a, s);
        case SC_ELEM_F16: return bias ? launch_route<SC_ELEM_F16, false, true>(a, s) : launch_route<SC_ELEM_F16, false, false>(a, s);
        default: return bias ? launch_route<SC_ELEM_BF16, false, true>(a, s) : launch_route<SC_ELEM_BF16, false, false>(a, s);
    }
}

extern "C" sc_status_t sparse_conv_route_experts_backward(const sc_route_experts_t* d, const void* x, const int32_t* ids, const float* dweights, void* dx, void* stream)
{
    const sc_status_t st = check(d, true);
    if (st != SC_OK) return st;
    if (d->T == 0) return SC_OK;
    if (!x || !ids || !dweights || !dx) return SC_ERR_NULL;
    if (!aligned(x, elem_bytes(d->x_type)) || !aligned(dx, elem_bytes(d->x_type)) || !aligned(ids, 4) || !aligned(dweights, 4)) return SC_ERR_UNSUPPORTED;
    RouteArgs a = args(d, x);
    a.ids_in = ids; a.dweights = dweights; a.dx = dx;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool whole = d->score == SC_SCORE_SOFTMAX && !d->normalize;
    switch (d->x_type) {
        case SC_ELEM_F32: return whole ? launch_route<SC_ELEM_F32, true, true>(a, s) : launch_route<SC_ELEM_F32, true, false>(a, s);
        case SC_ELEM_F16: return whole ? launch_route<SC_ELEM_F16, true, true>(a, s) : launch_route<SC_ELEM_F16, true, false>(a, s);
        default: return whole ? launch_route<SC_ELEM_BF16, true, true>(a, s) : launch_route<SC_ELEM_BF16, true, false>(a, s);
    }
}
