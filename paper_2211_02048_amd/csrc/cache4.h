// The cache of keys and values in 4 bits: layout, and the conversions that the store, the load and the attention share.
//
// A value is a four-bit float (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign) times a power of two that 32 channels of one head of
// one token have in common (e8m0: the byte s is 2^(s - 127)).  Two bits of significand times a power of two are exact in bf16 and,
// between 2^-24 and 49152, in fp16: what the matrix instructions multiply is what is held, with no further rounding.
// The cache is [head][keys, values][section]; a section holds the groups of 32 channels as planes [token][16 bytes], so that the
// tokens a wave reads lie side by side whatever the head size, then - where the last group has 16 channels or fewer - a plane
// [token][8 bytes], then the scales [token][1, 2, 4 or 8 bytes].
#pragma once

#include "common.h"

namespace sige {

struct Cache4Layout {
    long cap;           // tokens of a plane: the capacity rounded up to whole chunks of 32
    long section;       // bytes of a head's keys (or values)
    long scales;        // where a section's scales start
    int full, tail;     // planes of 32 channels; 1 if one of 16 follows
    int gs_log2;        // log2 of the scale bytes per token
};

inline Cache4Layout cache4_layout(int d, int capacity)
{
    Cache4Layout l;
    const int groups = (d + 31) / 32, rest = d % 32;
    l.tail = rest > 0 && rest <= 16;
    l.full = groups - l.tail;
    l.gs_log2 = groups <= 1 ? 0 : groups <= 2 ? 1 : groups <= 4 ? 2 : 3;
    l.cap = ((long)capacity + 31) / 32 * 32;
    l.scales = l.cap * (16 * l.full + 8 * l.tail);
    l.section = l.scales + (l.cap << l.gs_log2);
    return l;
}

// scale exponents that a store writes, by the rows' type: every value it stores is a finite number of that type
constexpr int CACHE4_E_MIN = -125, CACHE4_E_MAX = 125, CACHE4_F16_E_MIN = -23, CACHE4_F16_E_MAX = 13;
// scale bytes beyond these mark a group that is not finite (a store writes 255)
constexpr unsigned CACHE4_LAST = 127 + CACHE4_E_MAX, CACHE4_F16_LAST = 127 + CACHE4_F16_E_MAX;

__device__ __forceinline__ float cache4_scale(unsigned byte) { return __uint_as_float(byte << 23); }

// Two values (byte SEL of w: the even channel in its low four bits) as a pair of the compute type, even channel in the low half.
template <typename C, int SEL> __device__ __forceinline__ uint32_t cache4_pair(uint32_t w, float scale)
{
    if constexpr (sizeof(C) == 2 && __is_same(C, f16)) {
        union { decltype(__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(0u, 1.0f, 0)) v; uint32_t u; } r;
        r.v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, SEL);
        return r.u;
    } else {
        union { decltype(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(0u, 1.0f, 0)) v; uint32_t u; } r;
        r.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL);
        return r.u;
    }
}

// Eight values (four bytes) as a 16-byte vector of the compute type.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename C> __device__ __forceinline__ u32x4 cache4_eight(uint32_t w, float scale)
{
    return u32x4{cache4_pair<C, 0>(w, scale), cache4_pair<C, 1>(w, scale), cache4_pair<C, 2>(w, scale), cache4_pair<C, 3>(w, scale)};
}

}  // namespace sige
