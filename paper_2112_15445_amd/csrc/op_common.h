// What the operators of channels-last blocks share: element types, activations, 8-bit float codes and
// the checks of their arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "sparse_conv.h"

namespace sc {

constexpr int kQBlock = 128;                 // elements of a row that share a scale
constexpr float kCodeMax = 448.0f;           // largest 8-bit float (E4M3)
constexpr float kAmaxFloor = 0x1p-100f;      // smallest magnitude a block is scaled by: 448 / it is finite

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

template <int ET> struct ElemT;
template <> struct ElemT<SC_ELEM_F32> { using T = float; };
template <> struct ElemT<SC_ELEM_F16> { using T = _Float16; };
template <> struct ElemT<SC_ELEM_BF16> { using T = __bf16; };
template <> struct ElemT<SC_ELEM_E4M3> { using T = uint8_t; };
template <int ET> using Elem = typename ElemT<ET>::T;

inline int elem_bytes(int et) { return et == SC_ELEM_F32 ? 4 : et == SC_ELEM_E4M3 ? 1 : 2; }
inline bool is_wide(int et) { return et == SC_ELEM_F32 || et == SC_ELEM_F16 || et == SC_ELEM_BF16; }
inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// z / (1 + exp(-z)) within some 2 ulp of 32 bits, from e = exp(-|z|) <= 1, which overflows nothing: z / (1 + e), or z e / (1 + e) where z is
// negative.  e = 2^t for t = -|z| log2(e), with what rounding t left out (its own, and the constant's lower half) put back by 2^r = 1 + r ln 2; the
// reciprocal of 1 .. 2 with one step of Newton's.  |z| is cut off where e is 0 (an infinite one would make r a NaN); below -87.3, e and the result are 0.
// Group norm of 32 x 56x56 x 256 fp32 52 us, product 8192 x 4096 x 1024 -> fp32 85 (with expf and a division 57 and 94, as for 16 bits 48 and 81).
__device__ __forceinline__ float silu32(float z)
{
    constexpr float kLog2e = 0x1.715476p+0f, kLog2eLow = 0x1.4ae0c0p-26f, kLn2 = 0x1.62e430p-1f;
    const float m = -fminf(fabsf(z), 200.0f), t = m * kLog2e;
    const float r = fmaf(m, kLog2eLow, fmaf(m, kLog2e, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, r * kLn2, e);
    const float d = 1.0f + e;
    float inv = __builtin_amdgcn_rcpf(d);
    inv = fmaf(fmaf(-d, inv, 1.0f), inv, inv);
    return (z < 0.0f ? z * e : z) * inv;
}

// YT: type of the result.  What is rounded to 16 bits or to codes after SiLU takes the exponential through the product z log2(e), off by |z| 2^-23
// of the result (5e-6 at z = -40, where f16 rounds by 5e-4 of it), and a reciprocal right to one place (a scale of codes, 32 bits, is off by no more).
template <int ACT, int YT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == SC_ACT_RELU) return z < 0.0f ? 0.0f : z;      // (NaN stays NaN)
    else if constexpr (ACT == SC_ACT_SILU && YT == SC_ELEM_F32) return silu32(z);
    else if constexpr (ACT == SC_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    else return z;
}

// The code of t, |t| <= 448 but for the rounding of the scaling (which the comparison takes back).
__device__ __forceinline__ float code_range(float t) { return fabsf(t) > kCodeMax ? copysignf(kCodeMax, t) : t; }
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(code_range(a), code_range(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_range(c), code_range(d), v, true);
}
__device__ __forceinline__ uint8_t code1(float a)
{
    return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(code_range(a), 0.0f, 0, false);
}

// Sixteen bytes of x as floats: V values from any element-aligned address, or the first `have` of them and zeros behind.
template <int ET> constexpr int kVec = 16 / (int)sizeof(Elem<ET>);
template <int ET> __device__ __forceinline__ v4i load_raw(const Elem<ET>* x)
{
    v4i raw;
    __builtin_memcpy(&raw, x, 16);
    return raw;
}
// The same for what is read once: with the non-temporal hint (1 GiB is read at 7 TB/s with it and at 6 without).
template <int ET> __device__ __forceinline__ v4i load_raw_once(const Elem<ET>* x)
{
    typedef int any4i __attribute__((ext_vector_type(4), aligned(2)));
    return __builtin_nontemporal_load(reinterpret_cast<const any4i*>(x));
}
template <int ET> __device__ __forceinline__ v4i load_raw_part(const Elem<ET>* x, int have)
{
    Elem<ET> e[kVec<ET>];
    if (have <= 0) return v4i{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kVec<ET>; ++i) e[i] = x[min(i, have - 1)];       // (no branch a value: the loads go out together)
#pragma unroll
    for (int i = 0; i < kVec<ET>; ++i) e[i] = i < have ? e[i] : (Elem<ET>)0.0f;
    v4i raw;
    __builtin_memcpy(&raw, e, 16);
    return raw;
}
template <int ET> __device__ __forceinline__ void to_floats(v4i raw, float* f)
{
    typedef Elem<ET> vec __attribute__((ext_vector_type(kVec<ET>)));
    const vec v = __builtin_bit_cast(vec, raw);
#pragma unroll
    for (int i = 0; i < kVec<ET>; ++i) f[i] = (float)v[i];
}
// V floats rounded to the type, stored at any element-aligned address; the first `have` of them.
template <int ET, int V> __device__ __forceinline__ void store_vec(Elem<ET>* y, const float* f, int have)
{
    typedef Elem<ET> vec __attribute__((ext_vector_type(V)));
    vec v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (Elem<ET>)f[i];
    if (have >= V) __builtin_memcpy(y, &v, sizeof(v));
    else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < have) y[i] = v[i];
    }
}
// The same past the caches, for y on 16 bytes and whole.
template <int ET, int V> __device__ __forceinline__ void store_vec_past(Elem<ET>* y, const float* f)
{
    typedef Elem<ET> vec __attribute__((ext_vector_type(V)));
    vec v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (Elem<ET>)f[i];
    struct raw { v4i q[V * sizeof(Elem<ET>) / 16]; } r;
    __builtin_memcpy(&r, &v, sizeof(r));
#pragma unroll
    for (unsigned i = 0; i < sizeof(r) / 16; ++i) __builtin_nontemporal_store(r.q[i], reinterpret_cast<v4i*>(y) + i);
}
// The V codes of f * up; q on V bytes (zeros of f behind the end of a row become zero codes).
template <int V> __device__ __forceinline__ void store_codes(uint8_t* q, const float* f, float up)
{
    uint32_t w[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) w[i] = codes4(f[4 * i] * up, f[4 * i + 1] * up, f[4 * i + 2] * up, f[4 * i + 3] * up);
    if constexpr (V == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
}

// Sums and maxima over the sixteen lanes of a row: four rotations within the row, which the vector unit does by itself (a shuffle
// through LDS takes some 60 cycles each).
template <int N> __device__ __forceinline__ float row_ror(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum16(float v)
{
    v += row_ror<8>(v);
    v += row_ror<4>(v);
    v += row_ror<2>(v);
    return v + row_ror<1>(v);
}
__device__ __forceinline__ float max16(float v)
{
    v = fmaxf(v, row_ror<8>(v));
    v = fmaxf(v, row_ror<4>(v));
    v = fmaxf(v, row_ror<2>(v));
    return fmaxf(v, row_ror<1>(v));
}
__device__ __forceinline__ float sum64(float v)
{
    v = sum16(v);
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}
// ... over the L = 16 or 32 lanes that hold 128 values.
template <int L> __device__ __forceinline__ float max_block(float v)
{
    v = max16(v);
    if constexpr (L == 32) v = fmaxf(v, __shfl_xor(v, 16));
    return v;
}

inline sc_status_t launched() { return hipGetLastError() == hipSuccess ? SC_OK : SC_ERR_HIP; }

}  // namespace sc
