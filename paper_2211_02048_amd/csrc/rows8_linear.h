// What the kernels of the products of two matrices in 8 bits share: arguments, the step over a block of 128 channels, the gate.
#pragma once

#include <type_traits>

#include "rows8.h"

namespace sige {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Linear8Args {
    const unsigned char* x;
    const unsigned char* xs;
    const unsigned char* w;
    const unsigned char* ws;
    const float* bias;
    const void* base;
    void* y;
    unsigned char* q;
    unsigned char* s;
    Rows8 rows;
    int blocks;                 // of 128 input channels
    int Cout, x_ld, xs_ld, w_ld, ws_ld, base_ld, y_ld, q_ld, s_ld;
    int gate;
};

// n things in parts of `part`, the last one partly filled (in 64 bits: n + part - 1 need not fit an int).
inline long parts_of(int n, int part) { return ((long)n + part - 1) / part; }

// Lets a kernel have more LDS than 48 KB (one limit whatever the call, so that calls from two threads do not undo each other's).
inline int allow_lds(const char* who, const void* kern, int bytes)
{
    if (bytes <= 48 * 1024) return SIGE_OK;
    const hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    SIGE_REQUIRE(e == hipSuccess, SIGE_ERR_HIP, "%s: cannot reserve %d bytes of LDS: %s", who, bytes, hipGetErrorString(e));
    return SIGE_OK;
}

__device__ __forceinline__ i32x8 both(i32x4 a, i32x4 b) { return i32x8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}; }

// Eight codes times their scale as bf16 numbers (exact).
__device__ __forceinline__ bf16x8 expand8(int lo, int hi, float scale)
{
    union { decltype(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(0u, 1.0f, false)) v; int u; } p, q, r, t;
    p.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false);
    q.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
    r.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false);
    t.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
    return __builtin_bit_cast(bf16x8, i32x4{p.u, q.u, r.u, t.u});
}

__device__ __forceinline__ float finite_or_0(float f)
{
    const float m = fabsf(f);
    return m < __uint_as_float(0x7f800000u) ? m : 0.0f;
}

// The gated activation: u * gelu(g) or u * silu(g).  (Chosen per call, not per value: a choice between every two values keeps their chains from
// overlapping.)  gelu(g) = max(g, 0) - z erfc(z / sqrt 2) / 2 with z = |g|, which holds far below zero too, and
// erfc(z / sqrt 2) / 2 = t R(t) exp(-z^2 / 2) with t = 1 / (1 + z / 5): R is the polynomial of degree 6 whose largest relative
// error over 0 <= z <= 14 is smallest (1.2e-6 in 64 bits; fitted by linear programming).  In fp32 the largest error of gelu(g) relative to itself is
// 1.8e-6 down to g = -3; below, the rounding of the exponent adds z^2 2^-24: 2.1e-6 to -5, 3.8e-6 to -8, 6.0e-6 to -10, 7.2e-6 to -13 (gelu(-13)
// is 8e-38; from -13.2 on the result is 0).  For g > 0 1.6e-6 at most.  silu: 5.5e-7 down to g = -8, 3.9e-6 to -87; below, 0.  Both are a choice beside the half step
// 2^-4 of the codes.  The library's functions took five times as long as this: 23 us behind a tile of 256 x 256.
template <int GATE>
__device__ __forceinline__ float gate_value(float u, float g)
{
    if constexpr (GATE == SIGE_GATE_SILU) return u * (g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)));
    const float z = fabsf(g), t = __builtin_amdgcn_rcpf(fmaf(z, 0.2f, 1.0f));
    float r = fmaf(0.27912187576293945f, t, -0.3869353234767914f);
    r = fmaf(r, t, 0.4471128284931183f);
    r = fmaf(r, t, -0.12332696467638016f);
    r = fmaf(r, t, 0.13259808719158173f);
    r = fmaf(r, t, 0.07107879221439362f);
    r = fmaf(r, t, 0.0803513303399086f);
    const float tail = (z * t) * (r * __builtin_amdgcn_exp2f(z * (z * -0.72134752044448170f)));
    return u * (fmaxf(g, 0.0f) - tail);
}

}  // namespace sige
