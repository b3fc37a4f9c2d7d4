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

template <int ACT> __device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == SC_ACT_RELU) return z < 0.0f ? 0.0f : z;      // (NaN stays NaN)
    else if constexpr (ACT == SC_ACT_SILU) return z / (1.0f + __expf(-z));
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

inline sc_status_t launched() { return hipGetLastError() == hipSuccess ? SC_OK : SC_ERR_HIP; }

}  // namespace sc
