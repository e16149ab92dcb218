// sige_cache4_attn: attention of the edited query tokens on keys and values held in 4 bits (Sec. 3.2 "Extension to attention
// layers", Fig. "sige-attention": the queries of the edited tokens against all cached keys and values), the kernels.
//
// o_i = sum_t softmax_t(scale q_i . k_t) v_t over the tokens [begin_i, end_i) that the row sees.  As in sige_sparse_attn everything
// runs transposed, so that what belongs to a query stays in one lane (pair): S^T = K Q^T leaves the logits of a query in the
// registers of lanes l and l + 32, and the probabilities feed O^T += V^T P^T straight from there, because the order of the contraction
// is free as long as V^T is read in the same one.
//
// A cached value is exact in bf16 (fp16 queries: in fp16): sixteen conversions per 32 channels, the scale folded in by the
// instruction.  What differs by type is the other operand: bf16 and fp16 queries enter as they are; a single-precision
// query, and the probabilities beside it, as the sum of three bf16 numbers (24 bits), so that single precision runs on the bf16 matrix
// instructions at a third of their rate (the fp32 ones have a sixteenth) with exact products.
// A probability is rounded to the compute type once, by half a step at most (bf16 2^-8 of each, fp16 2^-11), without bias, and the
// denominator adds what was multiplied: through a column of ones beside V where the head size leaves one free, else as dot
// products of the rounded pairs with ones (single precision: the values themselves).  In bf16 this is a choice against two terms,
// hi + lo, which sige_sparse_attn feeds.  One term: the result is off by 2.2e-3 of itself (rms; its own rounding is 1.65e-3 of that, and
// what two terms come to).  Two terms: 34 % more time for 4096 queries of 16384 x 8 of 128 (274 -> 367 us), 27 - 37 % for 4096 of 4096 x
// 40 - 80, 7 % for one query of 65536.  The cached values themselves, with 2 bits of significand, put the result 0.17 of itself away
// from that on the rows that were stored.
//
// Two forms.  cache4_apart_kernel: every wave by itself, the waves of a workgroup share the keys out among them; no barrier until
// they meet.  cache4_common_kernel: four or eight waves of 32 queries each that expand every chunk once for all.  The vector instructions
// bound the first where there is work (per 64 keys x 32 queries x 64: about 90 for the expansion, 110 for the softmax), LDS and the order
// of the two kinds of instructions the second.  Measured: one query of 65536 x 8 of 64 in bf16 14.7 us (with the merge; 35.7 MB, 2.4 TB/s),
// 614 of 4096 x 8 of 80 in fp16 21 us (300 TFLOP/s: 160 workgroups of eight chunks per wave), 4096 of 16384 x 8 of 128 in bf16 265 - 302 us by
// card (1040 - 910 TFLOP/s; a library product reaches 1167).  Where the registers are bounded for more waves side by side some kernels keep a
// few values in scratch memory: heads of 33 to 64 with four waves per SIMD 1 and 17 registers, half-type heads of 193 to 224 2 and 9;
// single-precision heads of 225 to 256 66 and 96, all of a SIMD's.
#pragma once

#include "cache4.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace sige {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

struct Cache4AttnArgs {
    const void* q;
    const uint8_t* cache;
    void* o;
    float* ws;                 // partials [split][head][Nq][d + 4]: the d sums, the maximum, the denominator, 2 unused
    const int32_t* ranges;     // [Nq][2]: the tokens a row sees (NULL: all T)
    const int32_t* q_blocks;   // queries by block list, as sige_sparse_attn_blocks
    long section, cap, scales; // of Cache4Layout
    int q_ld, o_ld, Nq, T, heads, d;
    int splits, share;         // workgroups that share the tokens of a query out, and their chunks of all T
    int waves;                 // of a workgroup, where they share its tokens out: 1, 2, 4 or 8
    int full, gs_log2;
    float scale_log2e, inv_scale;  // and its inverse
    int q_tpb, q_bw, q_H, q_W;
    FastDiv d_heads, d_tpb, d_qbw, d_dq, d_splits;
};

template <typename T> struct Cache4Compute { typedef bf16 type; static constexpr int parts = 1; static constexpr unsigned last = CACHE4_LAST; };
template <> struct Cache4Compute<f16> { typedef f16 type; static constexpr int parts = 1; static constexpr unsigned last = CACHE4_F16_LAST; };
template <> struct Cache4Compute<float> { typedef bf16 type; static constexpr int parts = 3; static constexpr unsigned last = CACHE4_LAST; };

template <typename C> __device__ __forceinline__ void mma32(const u32x4& a, const u32x4& b, f32x16& c)
{
    if constexpr (__is_same(C, f16)) {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    } else {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
}

template <typename C> __device__ __forceinline__ uint32_t round2(float a, float b)
{
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    if constexpr (__is_same(C, f16)) {
        typedef _Float16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, v2));
    } else {
        typedef __bf16 v2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, v2));
    }
}

// Two floats as NP pairs of the compute type whose sums they are (to 8 NP bits of bf16).  ANY: of any size - single precision ends
// above bf16, where the first part is bf16's largest number instead of an infinity (what is infinite becomes NaN with the others).
template <typename C, int NP, bool ANY> __device__ __forceinline__ void split2(float a, float b, uint32_t (&out)[NP])
{
    constexpr float LARGEST = 0x1.fep127f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        if (ANY && i == 0) out[i] = round2<C>(fminf(fmaxf(a, -LARGEST), LARGEST), fminf(fmaxf(b, -LARGEST), LARGEST));
        else out[i] = round2<C>(a, b);
        if (i + 1 < NP) {
            a -= __uint_as_float(out[i] << 16);
            b -= __uint_as_float(out[i] & 0xffff0000u);
        }
    }
}

__device__ __forceinline__ long cache4_query_row(const Cache4AttnArgs& a, int qi)
{
    if (a.q_blocks == nullptr) return qi;
    int b, p, py, px;
    divmod(qi, a.d_tpb, b, p);
    divmod(p, a.d_qbw, py, px);
    const int y0 = a.q_blocks[2 * b], x0 = a.q_blocks[2 * b + 1];
    return (long)min(max(y0 + py, 0), a.q_H - 1) * a.q_W + min(max(x0 + px, 0), a.q_W - 1);
}

// The tokens that row qi sees, within [0, T).
__device__ __forceinline__ void cache4_range(const int32_t* ranges, int T, int qi, int& begin, int& end)
{
    begin = 0;
    end = T;
    if (ranges != nullptr) {
        begin = max(ranges[2 * (long)qi], 0);
        end = min(ranges[2 * (long)qi + 1], T);
    }
}

__device__ __forceinline__ int wave_min(int v)
{
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) v = min(v, __shfl_xor(v, x));
    return v;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_transposed(char* lds)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(__attribute__((address_space(3))) char*)lds);
}

// What the 32 rows of a wave see (one row per lane pair).  A row that sees nothing is left out of the bounds and written as zeros.
struct Cache4Seen {
    int begin, end;                // this lane's row
    bool none;
    int lo, hi;                    // the wave: the first token that some row sees, the end of the last one
    int lo_most, hi_least;         // the tokens between are seen by all rows
    __device__ __forceinline__ bool partial(int t0, int n) const { return t0 < lo_most || (long)t0 + n > hi_least; }
    // whether some row of this wave sees some of n tokens
    __device__ __forceinline__ bool any(long t0, int n) const { return __builtin_amdgcn_ballot_w64(!none && begin < t0 + n && end > t0) != 0ull; }
    // The chunks of n tokens of split z: an equal share of those between lo and hi, whatever part of the cache they are
    __device__ __forceinline__ void chunks(const Cache4AttnArgs& a, int n, int z, int& first, int& last) const
    {
        int c0 = 0, c1 = (int)(((long)hi + n - 1) / n), per = a.share;
        if (a.ranges != nullptr) {
            int rest;
            c0 = lo / n;
            c1 = max(c1, c0);
            divmod(c1 - c0 + a.splits - 1, a.d_splits, per, rest);
        }
        first = c0 + z * per;
        last = min(first + per, c1);
    }
};
__device__ __forceinline__ Cache4Seen cache4_seen(const Cache4AttnArgs& a, int qi)
{
    Cache4Seen s = {0, a.T, a.T == 0, 0, a.T, 0, a.T};
    if (a.ranges != nullptr) {
        if (qi < a.Nq) cache4_range(a.ranges, a.T, qi, s.begin, s.end);
        s.none = qi >= a.Nq || s.begin >= s.end;
        s.lo = __builtin_amdgcn_readfirstlane(wave_min(s.none ? a.T : s.begin));
        s.hi = __builtin_amdgcn_readfirstlane(-wave_min(s.none ? 0 : -s.end));
        s.lo_most = __builtin_amdgcn_readfirstlane(-wave_min(s.none ? 0 : -s.begin));
        s.hi_least = __builtin_amdgcn_readfirstlane(wave_min(s.none ? a.T : s.end));
    }
    return s;
}

// Q fragments (B operand of S^T = K Q^T) of row qi: step s holds 8 channels per lane.  HALVES: the lower lanes have the first 16
// channels of a group of 32 and the upper ones the others (a group takes two steps); else a step is 16 channels in their order.
template <typename T, int DT, bool ODD, bool HALVES, int NP>
__device__ __forceinline__ void cache4_queries(const Cache4AttnArgs& a, int qi, int head, int half, u32x4 (&qf)[NP][2 * DT - ODD])
{
    constexpr int DK = 2 * DT - ODD;
    using C = typename Cache4Compute<T>::type;
    const long qrow = cache4_query_row(a, min(qi, a.Nq - 1));
    const char* const qp = (const char*)a.q + (qrow * a.q_ld + (long)head * a.d) * (long)sizeof(T);
#pragma unroll
    for (int s = 0; s < DK; ++s) {
        const int dd = HALVES && !(ODD && s == DK - 1) ? 32 * (s >> 1) + 16 * half + 8 * (s & 1) : 16 * s + 8 * half;
#pragma unroll
        for (int p = 0; p < NP; ++p) qf[p][s] = u32x4{0u, 0u, 0u, 0u};
        if (qi < a.Nq && dd < a.d) {
            if constexpr (sizeof(T) == 4) {
                float f[8];
                unpack<float>(*(const uint4*)(qp + dd * 4), f);
                unpack<float>(*(const uint4*)(qp + dd * 4 + 16), f + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t w[NP];
                    split2<C, NP, true>(f[2 * j], f[2 * j + 1], w);
#pragma unroll
                    for (int p = 0; p < NP; ++p) qf[p][s][j] = w[p];
                }
            } else {
                qf[0][s] = *(const u32x4*)(qp + dd * 2);
            }
        }
    }
}

// Maxima from here on (of logits times log2 e): their rounding, which the fused operation of the exponents keeps, is no longer small
// beside the offset of fp16's probabilities (2^15, the type ends at 2^16), and from 2^31 on beside the range of single precision.
// (The test for it and a register take 0.8 % of 4096 queries of 16384 x 8 of 128, 270 -> 272 us, and nothing that shows elsewhere.)
constexpr float CACHE4_FAR = 1048576.0f;

// The sums of a wave's 32 rows.  Of a 32-key tile of logits a lane holds keys 8 * (r / 4) + 4 * half + r % 4 of its row.
template <typename T, int DT, bool ODD, int KT> struct Cache4Sums {
    using C = typename Cache4Compute<T>::type;
    static constexpr int NP = Cache4Compute<T>::parts;
    f32x16 o[DT];
    float m, l;
    unsigned lost;                 // groups of 32 channels in which the row sees a value that is no number

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int nt = 0; nt < DT; ++nt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[nt][r] = 0.0f;
        m = -INFINITY;
        l = 0.0f;
        lost = 0u;
    }
    // A chunk of which some row does not see everything: those logits are out.  marked: some value in it is no number (and counts 0 in
    // the products); the groups of those that the row sees are noted.  vscales: the scale bytes of the chunk's first value
    __device__ __forceinline__ void hide(const Cache4AttnArgs& a, const Cache4Seen& seen, int t0, int half, bool marked,
                                         const uint8_t* vscales, f32x16 (&sacc)[KT])
    {
        if (marked) {
#pragma unroll 1
            for (int i = 0; i < 16 * KT; ++i) {                    // (rolled: unrolled, its addresses took 60 registers)
                const int at = 8 * (i >> 2) + 4 * half + (i & 3);
                if (t0 + at < seen.begin || t0 + at >= seen.end) continue;
#pragma unroll 1
                for (int g = 0; g < DT; ++g)
                    if (vscales[(at << a.gs_log2) + g] > Cache4Compute<T>::last) lost |= 1u << g;
            }
        }
        const unsigned width = (unsigned)max(seen.end - seen.begin, 0), off = (unsigned)(t0 + 4 * half - seen.begin);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (off + (kt * 32 + 8 * (r >> 2) + (r & 3)) >= width) sacc[kt][r] = -INFINITY;
    }
    // After the last chunk: the noted groups of a row are NaN
    __device__ __forceinline__ void finish()
    {
        if (__builtin_amdgcn_ballot_w64(lost != 0u) == 0ull) return;
        const unsigned both = lost | (unsigned)__shfl_xor((int)lost, 32);
#pragma unroll
        for (int nt = 0; nt < DT; ++nt)
            if (both >> nt & 1u) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!(ODD && nt == DT - 1 && r >= 8)) o[nt][r] = NAN;
            }
    }
    // The running maximum, and the sums brought to it; returns what the exponents subtract.  Logits are compared raw: the scale
    // (> 0) goes into the exponent.
    __device__ __forceinline__ float settle(float scale_log2e, float inv_scale, f32x16 (&sacc)[KT])
    {
        float mr = sacc[0][0];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mr = fmaxf(mr, sacc[kt][r]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mr), __float_as_uint(mr), false, false);
        const float mx = fmaxf(m, fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * scale_log2e);
        const float m_at = mx == -INFINITY ? 0.0f : mx;            // (only tokens out of sight so far: nothing is subtracted)
        if (__builtin_amdgcn_ballot_w64(mx != m) != 0ull) {        // some row's maximum moved
            const float alpha = __builtin_amdgcn_exp2f(m - m_at);
            m = mx;
            l *= alpha;
#pragma unroll
            for (int nt = 0; nt < DT; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[nt][r] *= alpha;
        }
        // (fp16: probabilities times 2^15, numerator and denominator alike, so that those down to 2^-29 keep their 11 bits and
        // only what is below 2^-40 is lost)
        constexpr float up = __is_same(C, f16) ? 15.0f : 0.0f;
        float m_sub = m_at - up;
        if (__builtin_amdgcn_ballot_w64(fabsf(m_at) >= CACHE4_FAR) != 0ull) {
            // The products of such a row are rounded as its maximum was and its logits measured from there: the largest exponent is
            // exactly 0 (finite logits of 10^7 in fp16, of 2 10^9 in bf16 made infinite probabilities).  The other rows stay as they are.
            const bool mine = fabsf(m_at) >= CACHE4_FAR;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float e = sacc[kt][r] * scale_log2e;
                    asm volatile("" : "+v"(e));                    // (a product of its own, not a part of a fused operation)
                    sacc[kt][r] = mine ? (e - m_at) * inv_scale : sacc[kt][r];
                }
            m_sub = mine ? -up : m_sub;
        }
        return m_sub;
    }
    // The probabilities, and O^T += V^T P^T in steps of 16 keys; v(kt, s, nt): the V^T fragment.  URGENT: from the product on the wave
    // goes before the others of its SIMD (until its next softmax)
    template <bool URGENT, typename V> __device__ __forceinline__ void add(float scale_log2e, float m_sub, f32x16 (&sacc)[KT], V v)
    {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sacc[kt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[kt][r], scale_log2e, -m_sub));
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 pf[NP];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p0 = sacc[kt][8 * s + 2 * j], p1 = sacc[kt][8 * s + 2 * j + 1];
                    uint32_t w[NP];
                    split2<C, NP, false>(p0, p1, w);
#pragma unroll
                    for (int p = 0; p < NP; ++p) pf[p][j] = w[p];
                    if constexpr (!ODD) {
                        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
                        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                        if constexpr (NP > 1) l += p0 + p1;
                        else if constexpr (__is_same(C, f16)) l = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w[0]), __builtin_bit_cast(h2, 0x3c003c00u), l, false);
                        else l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, w[0]), __builtin_bit_cast(b2, 0x3f803f80u), l, false);
                    }
                }
                if (URGENT && kt == 0 && s == 0) __builtin_amdgcn_s_setprio(1);
                constexpr int TILES = DT > 6 ? 4 : DT;       // (fragments on their way: heads beyond 192 have no registers for all)
#pragma unroll
                for (int n0 = 0; n0 < DT; n0 += TILES) {
                    u32x4 vf[TILES];
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt)
                        if (n0 + nt < DT) vf[nt] = v(kt, s, n0 + nt);
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt)
                        if (n0 + nt < DT) {
#pragma unroll
                            for (int p = NP - 1; p >= 0; --p) mma32<C>(vf[nt], pf[p], o[n0 + nt]);       // (the small parts first)
                        }
                    if (TILES < DT) __builtin_amdgcn_sched_barrier(0);
                }
            }
    }
    // The denominator, in both lanes of a row
    __device__ __forceinline__ float total(int l32) const
    {
        if constexpr (ODD) return __shfl(o[DT - 1][8], l32);       // row 16 of the last tile: register 8 of the lower half
        else return l + __shfl_xor(l, 32);
    }
    // Four consecutive channels from dd on
    __device__ __forceinline__ float4 four(int nt, int rq) const
    {
        return make_float4(o[nt][4 * rq], o[nt][4 * rq + 1], o[nt][4 * rq + 2], o[nt][4 * rq + 3]);
    }
};

template <typename T> __device__ __forceinline__ void cache4_write(T* out, float4 v)
{
    if constexpr (sizeof(T) == 4) *(float4*)out = v;
    else *(uint2*)out = make_uint2(round2<T>(v.x, v.y), round2<T>(v.z, v.w));
}

// ---- every wave by itself ----------------------------------------------------------------------------------------------------

// 32-key tiles per chunk, by what their logits take in registers
constexpr int cache4_apart_tiles(int DT, int parts) { return DT <= (parts > 1 ? 2 : 3) ? 2 : 1; }
constexpr int cache4_apart_bytes(int DT, int parts) { return 32 * cache4_apart_tiles(DT, parts) * 64 * DT; }     // a chunk's V rows in LDS
// waves of a workgroup: what their sums take in LDS when they meet
constexpr int cache4_apart_waves(int DT, int parts) { return DT <= (parts > 1 ? 2 : 4) ? 8 : 4; }
// waves per SIMD: their registers hold the next chunk beside everything, and the waves of one workgroup are two per SIMD anyway
constexpr int cache4_apart_side(int DT, int parts) { return parts > 1 ? (DT <= 3 ? 2 : 1) : DT <= 7 ? 2 : 1; }
// Many queries, half types.  Heads up to 64: four waves per SIMD, two workgroups side by side (4096 queries of 4096 x 8 of 64 74 -> 64 us,
// of 40 62 -> 50; one query of 65536 keys 15.1 -> 16.1).  Larger heads have no registers for that: the common form.  For heads up to 64
// the common form wins on long caches alone (bf16, us, this one | common chunks: 4096 of 16384 x 8 of 64 202 | 180, of 40 162 | 153; 4096 of 4096
// x 64 61 | 61, x 40 46 | 51, x 32 36 | 44; 2048 of 4096 x 64 32 | 42; 1500 of 1500 x 64 16 | 29; 4096 of 1024 x 32 12 | 23) and is not built.
constexpr bool cache4_crowds(int DT, int parts) { return parts == 1 && DT <= 2; }
constexpr int CACHE4_CROWD_WAVES = 4;              // of a workgroup (eight: 1500 queries of 1500 x 8 of 64 18.4 -> 19.2 us)
constexpr bool cache4_has_common(int DT, int parts) { return parts == 1 && DT > 2; }
// The 64 bytes of group g of a V row: which of the row's groups of 64 bytes holds it.  Four neighbouring keys keep a group on
// different banks, in the writes (a lane per key) and in the transposed reads (four keys per 16 lanes).
template <int DT> __device__ __forceinline__ int cache4_apart_group(int key, int g)
{
    return DT % 2 ? g : DT % 4 ? g ^ ((key >> 1) & 1) : g ^ (key & 3);
}

// DT = 32-wide tiles over d; ODD: the last one has 16 channels (d % 32 is 8 or 16), and its row 16 is the row of ones.
// The waves of a workgroup (up to NK) have the same 32 queries and take every waves-th chunk of the tokens.  K goes from memory straight into the
// first product's operands (8 bytes of a key and group per lane: the order of the channels is the queries' too), V through the
// wave's own rows in LDS, which it is transposed out of.  WAVES: per SIMD, whose registers they share.
template <typename T, int DT, bool ODD, int NK, int WAVES>
__global__ __launch_bounds__(64 * NK, WAVES) void cache4_apart_kernel(Cache4AttnArgs a)
{
    using C = typename Cache4Compute<T>::type;
    constexpr int NP = Cache4Compute<T>::parts;
    constexpr unsigned LAST = Cache4Compute<T>::last;
    constexpr int KT = cache4_apart_tiles(DT, NP), KCH = 32 * KT;
    constexpr int VROW = 64 * DT;
    constexpr int DK = 2 * DT - ODD;               // 16-wide steps over d for S^T
    constexpr int VU = KT == 2 ? DT : (DT + 1) / 2;        // groups a lane expands per chunk: of one of 64 keys, or every other one of 32
    constexpr int SW = (DT + 3) / 4;               // words of a token's scales
    constexpr int GS = DT == 1 ? 1 : DT == 2 ? 2 : DT <= 4 ? 4 : 8;
    extern __shared__ uint4 lds4[];
    char* const lds = reinterpret_cast<char*>(lds4);
    const int d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int qt, head;                                  // (the heads side by side: with eight of them each XCD keeps one in its L2)
    divmod((int)blockIdx.x, a.d_heads, qt, head);
    const int qi = qt * 32 + l32;
    const Cache4Seen seen = cache4_seen(a, qi);
    const int waves = a.waves;
    int c, c_end;
    seen.chunks(a, KCH, blockIdx.z, c, c_end);
    c += wave;
    if (a.ranges != nullptr)                       // (between the parts that the rows see there may be chunks that none does)
        while (c < c_end && !seen.any((long)c * KCH, KCH)) c += waves;

    char* const vs = lds + wave * cache4_apart_bytes(DT, NP);
    const uint8_t* const ksec = a.cache + 2L * head * a.section;
    const uint8_t* const vsec = ksec + a.section;

    // a chunk on its way: of K, this lane's half of the groups of keys l32 (and l32 + 32); of V, the groups of a key
    u32x2 kc[KT][DT];
    u32x4 vc[VU];
    uint32_t ksc[KT][SW], vsc[SW];
    const int vkey = KT == 2 ? lane : l32;
    auto scales = [&](const uint8_t* p, uint32_t (&w)[SW]) {
        if constexpr (DT == 1) w[0] = *p;
        else if constexpr (DT == 2) w[0] = *(const uint16_t*)p;
        else if constexpr (DT <= 4) w[0] = *(const uint32_t*)p;
        else { const u32x2 v = *(const u32x2*)p; w[0] = v.x; w[SW - 1] = v.y; }
    };
    auto fetch = [&](int c) {
        const long t0 = (long)c * KCH;
        const int last = (int)min((long)KCH, (long)a.T - t0) - 1;   // (tokens past the end: the last one again)
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const unsigned key = (unsigned)min(kt * 32 + l32, last);
#pragma unroll
            for (int g = 0; g < DT; ++g) {
                if (ODD && g == DT - 1) kc[kt][g] = u32x2{*(const uint32_t*)(ksec + (a.full * a.cap * 16 + t0 * 8) + (key * 8u + half * 4u)), 0u};
                else kc[kt][g] = *(const u32x2*)(ksec + (g * a.cap * 16 + t0 * 16) + (key * 16u + half * 8u));
            }
            scales(ksec + (a.scales + t0 * GS) + key * (unsigned)GS, ksc[kt]);
        }
        const unsigned key = (unsigned)min(vkey, last);
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int g = KT == 2 ? u : 2 * u + half;
            if (KT == 1 && 2 * u + 1 >= DT && half) break;          // (an odd number of groups: the last one is the lower half's)
            if (ODD && (KT == 2 ? u == DT - 1 : 2 * u + 1 >= DT - 1 && g == DT - 1)) {
                const u32x2 w = *(const u32x2*)(vsec + (a.full * a.cap * 16 + t0 * 8) + key * 8u);
                vc[u] = u32x4{w.x, w.y, 0u, 0u};
            } else {
                vc[u] = *(const u32x4*)(vsec + (g * a.cap * 16 + t0 * 16) + key * 16u);
            }
        }
        scales(vsec + (a.scales + t0 * GS) + key * (unsigned)GS, vsc);
    };
    // a group's scale; one that is no number is the power of two that the conversion makes NaN of (or 0, see below)
    auto scale_of = [&](uint32_t word, int shift, unsigned bad) {
        const unsigned byte = (word >> shift) & 255u;
        return __uint_as_float(byte > LAST ? bad : byte << 23);
    };
    if (c < c_end) fetch(c);
    u32x4 qf[NP][DK];
    cache4_queries<T, DT, ODD, true>(a, qi, head, half, qf);

    // V rows: the 16-byte vectors of a group lie in the order of their number ^ ((key >> 2) & 3), for the banks of the writes
    auto v_at = [&](int key, int g, int j) { return key * VROW + cache4_apart_group<DT>(key, g) * 64 + ((j ^ ((key >> 2) & 3)) * 16); };
    if constexpr (ODD) {                           // the columns that no group fills (row 16 of the last tile: ones)
        constexpr uint32_t ONE = __is_same(C, f16) ? 0x3c00u : 0x3f80u;
        for (int j = lane; j < KCH * 2; j += 64) *(u32x4*)(vs + v_at(j >> 1, DT - 1, 2 + (j & 1))) = u32x4{j & 1 ? 0u : ONE, 0u, 0u, 0u};
    }
    // where this lane's share of a transposed read starts: four lanes take the 16 columns of one key, four keys per 16 lanes,
    // lane i of the 16 receives column i of the four keys.  (The keys of one lane differ by multiples of 8: one more turn of 2
    // in the order of the vectors for every 8.)
    const int rkey = 4 * half + ((lane & 15) >> 2), rvec = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    int r_lo[DT % 2 ? 1 : DT];                     // by tile (an odd number of them: the tiles follow each other)
#pragma unroll
    for (int nt = 0; nt < (DT % 2 ? 1 : DT); ++nt) r_lo[nt] = v_at(rkey, nt, rvec) + (lane & 1) * 8;
    const int r_up = ((rvec ^ half ^ 2) - (rvec ^ half)) * 16;      // what the vector's place differs by 8 keys on
    auto v_fragment = [&](int kt, int s, int nt) {
        char* const at = vs + (kt * 32 + 16 * s) * VROW + (DT % 2 ? r_lo[0] + nt * 64 : r_lo[nt]);
        union { s16x4 h[2]; u32x4 u; } vf;
        vf.h[0] = read_transposed(at);
        vf.h[1] = read_transposed(at + 8 * VROW + r_up);
        return vf.u;
    };

    Cache4Sums<T, DT, ODD, KT> sums;
    sums.clear();
    while (c < c_end) {
        const int t0 = c * KCH;
        int next = c + waves;
        if (a.ranges != nullptr)
            while (next < c_end && !seen.any((long)next * KCH, KCH)) next += waves;
        // In a chunk of which some row does not see everything a value that is no number counts 0 - a probability of 0 times NaN
        // is NaN -, and the rows that see it are marked below.
        const bool partial = seen.partial(t0, KCH);
        const unsigned bad_v = partial ? 0u : 0x7f800000u;
        bool marked = false;
        if (partial) {
#pragma unroll
            for (int g = 0; g < DT; ++g) marked |= ((vsc[g >> 2] >> (8 * (g & 3))) & 255u) > LAST;
            marked = __builtin_amdgcn_ballot_w64(marked) != 0ull;
        }
        // V rows (LDS operations of a wave stay in order: the last chunk's reads are behind it)
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int g = KT == 2 ? u : 2 * u + half;
            const float scale = scale_of(vsc[(KT == 2 ? u : 2 * u) >> 2], KT == 2 ? 8 * (u & 3) : 16 * (u & 1) + 8 * half, bad_v);
            const bool tail = ODD && (KT == 2 ? u == DT - 1 : 2 * u + 1 >= DT - 1 && g == DT - 1);
            u32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = cache4_eight<C>(vc[u][j], scale);
            if (KT == 1 && 2 * u + 1 >= DT && half) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!(tail && j >= 2)) *(u32x4*)(vs + v_at(vkey, g, j)) = x[j];
        }
        // S^T: rows = keys, columns = queries
        f32x16 sacc[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[kt][r] = 0.0f;
#pragma unroll
        for (int s = 0; s < DK; ++s)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const int g = s >> 1;
                const u32x4 kf = cache4_eight<C>(kc[kt][g][s & 1], scale_of(ksc[kt][g >> 2], 8 * (g & 3), 0x7f800000u));
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) mma32<C>(kf, qf[p][s], sacc[kt]);      // (the small parts first)
            }
        if (next < c_end) fetch(next);             // in flight during the softmax and the second product
        if (partial) sums.hide(a, seen, t0, half, marked, vsec + a.scales + (long)t0 * GS, sacc);
        const float m_sub = sums.settle(a.scale_log2e, a.inv_scale, sacc);
        sums.template add<false>(a.scale_log2e, m_sub, sacc, v_fragment);
        c = next;
    }

    // the waves' shares of the tokens, brought to a common maximum and added in wave order
    sums.finish();
    float l_tot = sums.total(l32);
    if (seen.none) { sums.m = -INFINITY; l_tot = 0.0f; }            // (what such a row added up is not read)
    float* const comb = reinterpret_cast<float*>(lds);              // [NK][32 queries][d sums, maximum, denominator, 2 unused]
    const int cs = d + 4;
    __syncthreads();                                                // (chunks no longer needed)
    {
        float* const mine = comb + (wave * 32 + l32) * cs;
        if (qi < a.Nq) {                                            // (few queries: few rows to bring together)
            if (half == 0) *(float2*)(mine + d) = make_float2(sums.m, l_tot);
#pragma unroll
            for (int nt = 0; nt < DT; ++nt)
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) {
                    const int dd = nt * 32 + 8 * rq + 4 * half;
                    if (dd < d) *(float4*)(mine + dd) = sums.four(nt, rq);
                }
        }
    }
    __syncthreads();
    const int dq = d >> 2, todo = min(32, a.Nq - qt * 32) * dq;
    auto meet = [&](auto count) {
        constexpr int N = decltype(count)::value;
        for (int e = tid; e < todo; e += 64 * N) {
            int q, g;
            divmod(e, a.d_dq, q, g);
            const int qq = qt * 32 + q;
            const float* const src = comb + q * cs;
            float m = -INFINITY, den = 0.0f;
            float4 num = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < N; ++w) m = fmaxf(m, src[w * 32 * cs + d]);
#pragma unroll
            for (int w = 0; w < N; ++w) {
                const float2 ml = *(const float2*)(src + w * 32 * cs + d);
                const float4 v = *(const float4*)(src + w * 32 * cs + 4 * g);
                // (a wave without keys carries -inf, 0 and zeros; one whose values hold a NaN keeps it whatever its weight)
                const float f = ml.x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml.x - m);
                den += ml.y * f;
                num.x += v.x * f; num.y += v.y * f; num.z += v.z * f; num.w += v.w * f;
            }
            int b, en;
            cache4_range(a.ranges, a.T, qq, b, en);
            if (b >= en) num = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (a.splits == 1) {
                const float inv = b >= en ? 0.0f : 1.0f / den;
                cache4_write((T*)a.o + (long)qq * a.o_ld + head * d + 4 * g, make_float4(num.x * inv, num.y * inv, num.z * inv, num.w * inv));
            } else {
                float* const w = a.ws + (((long)blockIdx.z * a.heads + head) * a.Nq + qq) * (d + 4);
                *(float4*)(w + 4 * g) = num;
                if (g == 0) *(float2*)(w + d) = make_float2(m, den);
            }
        }
    };
    if (waves == NK) meet(std::integral_constant<int, NK>());
    else if (waves == 1) meet(std::integral_constant<int, 1>());
    else if (waves == 2 || NK == 4) meet(std::integral_constant<int, 2>());
    else meet(std::integral_constant<int, NK == 4 ? 2 : 4>());
}

// ---- waves on the same chunks (half types) -----------------------------------------------------------------------------------

// Waves of a workgroup.  Heads up to 96: four, three workgroups per compute unit.  Larger ones: eight, which halves what a query pays for the
// expansion (4096 queries of 16384 x 8 of 128 327 -> 298 us, 1024 of 16384 x 128 102 -> 93, 2048 of 4096 x 160 81 -> 76, 1024 of 4096 x 256
// 82 both; 4096 of 4096 x 80 78 against 70 with four).
constexpr int cache4_common_waves(int DT) { return DT <= 3 ? 4 : 8; }
constexpr int cache4_common_tiles(int DT) { return DT <= 4 ? 2 : 1; }                    // 32-key tiles per chunk
// bytes between V rows in LDS: an odd multiple of 64, so that the keys of a transposed read fall on different banks; between K rows:
// 16 bytes more than the channels
constexpr int cache4_common_v_row(int DT) { return 64 * (DT | 1); }
constexpr int cache4_common_k_row(int DT, bool ODD) { return 32 * (2 * DT - ODD) + 16; }
constexpr int cache4_common_bytes(int DT, bool ODD) { return 32 * cache4_common_tiles(DT) * (cache4_common_v_row(DT) + cache4_common_k_row(DT, ODD)); }

// The waves have 32 queries each and expand every chunk once for all, K and V rows of the compute type in LDS: the next chunk into one
// buffer while the other is multiplied, one barrier per chunk.  The registers are bounded for two waves per SIMD: told so, the
// compiler keeps heads up to 128 in half of what it takes otherwise (with four waves, 4096 queries of 16384 x 8 of 128 580 -> 367 us, 2048
// of 4096 x 160 146 -> 85, 1024 of 4096 x 256 125 -> 77).
template <typename T, int DT, bool ODD>
__global__ __launch_bounds__(64 * cache4_common_waves(DT), 2) void cache4_common_kernel(Cache4AttnArgs a)
{
    using C = typename Cache4Compute<T>::type;
    constexpr int NW = cache4_common_waves(DT);
    constexpr unsigned LAST = Cache4Compute<T>::last;
    constexpr int KT = cache4_common_tiles(DT), KCH = 32 * KT;
    constexpr int VROW = cache4_common_v_row(DT), KROW = cache4_common_k_row(DT, ODD), CHUNK = cache4_common_bytes(DT, ODD);
    constexpr int DK = 2 * DT - ODD;               // 16-wide steps over d for S^T
    constexpr int UNITS = KT == 2 ? 2 * DT : DT;   // what a wave expands at a time: 64 groups of 32 channels
    constexpr int NU = (UNITS + NW - 1) / NW;
    extern __shared__ uint4 lds4[];
    __shared__ int marked_chunk[2];                // the chunk (+ 1) that left a value that is no number out of a buffer
    __shared__ int ends[NW][4];
    char* const lds = reinterpret_cast<char*>(lds4);
    const int d = a.d;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int qt, head;                                  // (the heads side by side: with eight of them each XCD keeps one in its L2)
    divmod((int)blockIdx.x, a.d_heads, qt, head);
    const int qi = (qt * NW + wave) * 32 + l32;
    const bool q_ok = qi < a.Nq;
    Cache4Seen seen = cache4_seen(a, qi);
    if (tid < 2) marked_chunk[tid] = 0;
    if (a.ranges != nullptr) {                     // what the workgroup's rows see
        if (lane == 0) { ends[wave][0] = seen.lo; ends[wave][1] = seen.hi; ends[wave][2] = seen.lo_most; ends[wave][3] = seen.hi_least; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            seen.lo = min(seen.lo, ends[w][0]);
            seen.hi = max(seen.hi, ends[w][1]);
            seen.lo_most = max(seen.lo_most, ends[w][2]);
            seen.hi_least = min(seen.hi_least, ends[w][3]);
        }
        seen.lo = __builtin_amdgcn_readfirstlane(seen.lo);
        seen.hi = __builtin_amdgcn_readfirstlane(seen.hi);
        seen.lo_most = __builtin_amdgcn_readfirstlane(seen.lo_most);
        seen.hi_least = __builtin_amdgcn_readfirstlane(seen.hi_least);
    } else {
        __syncthreads();
    }
    int c, c_end;
    seen.chunks(a, KCH, blockIdx.z, c, c_end);
    const uint8_t* const sec = a.cache + 2L * head * a.section;

    // a unit's 64 groups: of 64 keys (K's units, then V's), or of the keys and the values of 32
    u32x4 code[NU];
    unsigned sbyte[NU];
    auto fetch = [&](int c) {
        const long t0 = (long)c * KCH;
        const int last = (int)min((long)KCH, (long)a.T - t0) - 1;   // (tokens past the end: the last one again)
        const unsigned key = (unsigned)min(KT == 2 ? lane : l32, last);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = wave + NW * i;
            if (UNITS % NW != 0 && u >= UNITS) break;
            const int g = KT == 2 && u >= DT ? u - DT : u;
            const uint8_t* const base = sec + ((KT == 2 ? u >= DT : half) ? a.section : 0);
            if (ODD && g == DT - 1) {
                const u32x2 w = *(const u32x2*)(base + (a.full * a.cap * 16 + t0 * 8) + key * 8u);
                code[i] = u32x4{w.x, w.y, 0u, 0u};
            } else {
                code[i] = *(const u32x4*)(base + (g * a.cap * 16 + t0 * 16) + key * 16u);
            }
            sbyte[i] = (base + (a.scales + (t0 << a.gs_log2)) + g)[key << a.gs_log2];
        }
    };
    // the expanded units' rows in a buffer (K rows, then V rows)
    auto stage = [&](int c, int buf) {
        const bool partial = seen.partial(c * KCH, KCH);
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = wave + NW * i;
            if (UNITS % NW != 0 && u >= UNITS) break;
            const int g = KT == 2 && u >= DT ? u - DT : u;
            const int which = KT == 2 ? u >= DT : half;
            const int key = KT == 2 ? lane : l32;
            const bool tail = ODD && g == DT - 1;
            char* const dst = lds + buf * CHUNK + (which ? KCH * KROW + key * VROW : key * KROW) + g * 64;
            // a group that is no number: NaN for all who see it; a value in a chunk of which some row does not see everything: 0 - a
            // probability of 0 times NaN is NaN -, and the rows that see it are marked below
            const bool bad = sbyte[i] > LAST;
            const float scale = __uint_as_float(bad ? (which && partial ? 0u : 0x7f800000u) : sbyte[i] << 23);
            if (partial && bad && which) marked_chunk[buf] = c + 1;
            // V rows lie an odd multiple of 64 bytes apart, four lanes on the banks of one: every four lanes start with another of their
            // group's four vectors (else the writes took 60 of the 110 cycles that LDS was busy per chunk, 4096 queries of 16384 x 128)
            u32x4 w = code[i];
            int turn = 0;
            if (which && !tail) {
                turn = (key >> 2) & 3;
                if (turn & 1) w = u32x4{w.y, w.z, w.w, w.x};
                if (turn & 2) w = u32x4{w.z, w.w, w.x, w.y};
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!(tail && j >= 2)) *(u32x4*)(dst + 16 * ((j + turn) & 3)) = cache4_eight<C>(w[j], scale);
        }
    };
    if (c < c_end) fetch(c);
    u32x4 qf[1][DK];
    cache4_queries<T, DT, ODD, false>(a, qi, head, half, qf);
    if constexpr (ODD) {                           // the columns of the V rows that no group fills (row 16 of the last tile: ones)
        constexpr uint32_t ONE = __is_same(C, f16) ? 0x3c00u : 0x3f80u;
        for (int j = tid; j < 2 * KCH * 2; j += 64 * NW) {
            const int buf = j / (KCH * 2), key = (j >> 1) % KCH;
            *(u32x4*)(lds + buf * CHUNK + KCH * KROW + key * VROW + (DT - 1) * 64 + 32 + (j & 1) * 16) = u32x4{j & 1 ? 0u : ONE, 0u, 0u, 0u};
        }
    }
    // where this lane's share of a transposed read starts: four lanes take the 16 columns of one key, four keys per 16 lanes,
    // lane i of the 16 receives column i of the four keys
    const int tr = KCH * KROW + (4 * half + ((lane & 15) >> 2)) * VROW + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;

    Cache4Sums<T, DT, ODD, KT> sums;
    sums.clear();
    if (c < c_end) {
        stage(c, 0);
        if (c + 1 < c_end) fetch(c + 1);
    }
    for (int buf = 0; c < c_end; ++c, buf ^= 1) {
        __syncthreads();                           // this chunk's rows are there, the other buffer's have been read
        if (c + 1 < c_end) {
            stage(c + 1, buf ^ 1);
            if (c + 2 < c_end) fetch(c + 2);
        }
        const int t0 = c * KCH;
        char* const rows = lds + buf * CHUNK;
        // Of the two waves on a SIMD the one in its softmax yields to the other, from here to the logits and again from the second
        // product to the next chunk's rows (4096 queries of 16384 x 8 of 128 299.5 -> 293 us, 2048 of 4096 x 160 78.8 -> 75.7; the softmax
        // first 299)
        __builtin_amdgcn_s_setprio(1);
        f32x16 sacc[KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[kt][r] = 0.0f;
            constexpr int AT_ONCE = DK > 14 ? 8 : DK;       // (K fragments on their way: heads of 256 have no registers for all)
#pragma unroll
            for (int s0 = 0; s0 < DK; s0 += AT_ONCE) {
                u32x4 kf[AT_ONCE];
#pragma unroll
                for (int s = 0; s < AT_ONCE; ++s)
                    if (s0 + s < DK) kf[s] = *(const u32x4*)(rows + (kt * 32 + l32) * KROW + (16 * (s0 + s) + 8 * half) * 2);
#pragma unroll
                for (int s = 0; s < AT_ONCE; ++s)
                    if (s0 + s < DK) mma32<C>(kf[s], qf[0][s0 + s], sacc[kt]);
                if (AT_ONCE < DK) __builtin_amdgcn_sched_barrier(0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if (seen.partial(t0, KCH))
            sums.hide(a, seen, t0, half, __builtin_amdgcn_readfirstlane(marked_chunk[buf]) == c + 1,
                      sec + a.section + a.scales + ((long)t0 << a.gs_log2), sacc);
        const float m_sub = sums.settle(a.scale_log2e, a.inv_scale, sacc);
        sums.template add<true>(a.scale_log2e, m_sub, sacc, [&](int kt, int s, int nt) {
            char* const at = rows + tr + (kt * 32 + 16 * s) * VROW + nt * 64;
            union { s16x4 h[2]; u32x4 u; } vf;
            vf.h[0] = read_transposed(at);
            vf.h[1] = read_transposed(at + 8 * VROW);
            return vf.u;
        });
    }

    sums.finish();
    float l_tot = sums.total(l32);
    if (!q_ok) return;
    if (seen.none) { sums.m = -INFINITY; l_tot = 0.0f; }
    const float inv = seen.none ? 0.0f : 1.0f / l_tot;
    float* const w = a.ws + (((long)blockIdx.z * a.heads + head) * a.Nq + qi) * (d + 4);
    if (a.splits > 1 && half == 0) *(float2*)(w + d) = make_float2(sums.m, l_tot);
#pragma unroll
    for (int nt = 0; nt < DT; ++nt)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
            const int dd = nt * 32 + 8 * rq + 4 * half;
            if (dd >= d) continue;
            float4 v = sums.four(nt, rq);
            if (seen.none) v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);          // (what such a row added up is not read)
            if (a.splits == 1) cache4_write((T*)a.o + (long)qi * a.o_ld + head * d + dd, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
            else *(float4*)(w + dd) = v;
        }
}

// ---- the splits' partial results ---------------------------------------------------------------------------------------------

// Added in their order: four consecutive channels of a (query, head) per P neighbouring lanes.
template <typename T, int P>
__global__ __launch_bounds__(256) void cache4_merge_kernel(Cache4AttnArgs a)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    const int d = a.d, dq = d >> 2, sub = (int)(i % P);
    const long grp = i / P;
    const bool live = grp < (long)a.Nq * a.heads * dq;      // (whole groups: P divides the workgroup size)
    const long gi = live ? grp : 0;
    const long qh = gi / dq;
    const int dd = (int)(gi - qh * dq) * 4, head = (int)(qh % a.heads), qi = (int)(qh / a.heads);
    const long apart = (long)a.heads * a.Nq * (d + 4);
    const float* const w0 = a.ws + ((long)head * a.Nq + qi) * (d + 4);
    constexpr int B = 4;                                    // splits per lane, at most
    float2 ml[B];
    float4 val[B];
#pragma unroll
    for (int j = 0; j < B; ++j) {
        const float* const w = w0 + min(sub + j * P, a.splits - 1) * apart;
        ml[j] = *(const float2*)(w + d);
        val[j] = *(const float4*)(w + dd);
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < B; ++j)
        if (sub + j * P < a.splits) m = fmaxf(m, ml[j].x);
#pragma unroll
    for (int x = 1; x < P; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
    float den = 0.0f, num[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < B; ++j) {
        if (sub + j * P >= a.splits) continue;
        const float f = ml[j].x == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ml[j].x - m);
        den += ml[j].y * f;
        num[0] += val[j].x * f; num[1] += val[j].y * f; num[2] += val[j].z * f; num[3] += val[j].w * f;
    }
#pragma unroll
    for (int x = 1; x < P; x <<= 1) {                       // (a sum of two is the same in both partners)
        den += __shfl_xor(den, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += __shfl_xor(num[e], x);
    }
    if (!live || sub != 0) return;
    int b, en;
    cache4_range(a.ranges, a.T, qi, b, en);
    const float inv = 1.0f / den;
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] = b >= en ? 0.0f : num[e] * inv;
    cache4_write((T*)a.o + (long)qi * a.o_ld + head * d + dd, make_float4(num[0], num[1], num[2], num[3]));
}

// How a call is cut (cache4_attn.hip), and its launch, one file per type.
struct Cache4Form { bool many; int splits; };                // many: enough queries for the form that takes them
int launch_cache4_f32(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st);
int launch_cache4_f16(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st);
int launch_cache4_bf16(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st);

template <typename T, int DT, bool ODD>
static int launch_cache4_as(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st)
{
    constexpr int NP = Cache4Compute<T>::parts, NK = cache4_apart_waves(DT, NP);
    void (*kern)(Cache4AttnArgs) = cache4_apart_kernel<T, DT, ODD, NK, cache4_apart_side(DT, NP)>;
    int rows = 32, threads = 64 * a.waves;
    size_t lds = a.waves * std::max((size_t)cache4_apart_bytes(DT, NP), 32 * (a.d + 4) * sizeof(float));
    if constexpr (cache4_crowds(DT, NP))
        if (f.many) kern = cache4_apart_kernel<T, DT, ODD, CACHE4_CROWD_WAVES, 4>;
    if constexpr (cache4_has_common(DT, NP))
        if (f.many) {
            kern = cache4_common_kernel<T, DT, ODD>;
            rows = 32 * cache4_common_waves(DT);
            threads = 64 * cache4_common_waves(DT);
            lds = 2 * (size_t)cache4_common_bytes(DT, ODD);
        }
    const long tiles = ((long)a.Nq + rows - 1) / rows * a.heads, groups = (long)a.Nq * a.heads * (a.d / 4);
    const int P = a.splits <= 4 ? 1 : a.splits <= 16 ? 4 : 16;             // (at most 64 splits)
    SIGE_REQUIRE(tiles * a.splits * threads < (1L << 32) && (a.splits == 1 || groups * P < (1L << 32) - 256), SIGE_ERR_UNSUPPORTED,
                 "sige_cache4_attn: too many queries");                       // (what a launch can have of threads)
    if (lds > 48 * 1024) {                         // (allowed: the same for all calls of a kernel, two may be made at once)
        const size_t most = std::max(lds, NK * std::max((size_t)cache4_apart_bytes(DT, NP), 32 * (32 * DT + 4) * sizeof(float)));
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)most);
        SIGE_REQUIRE(e == hipSuccess, SIGE_ERR_HIP, "sige_cache4_attn: cannot reserve %zu bytes of LDS: %s", lds, hipGetErrorString(e));
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles, 1, a.splits), dim3(threads), lds, st, a);
    SIGE_LAUNCH_CHECK("sige_cache4_attn");
    if (a.splits == 1) return SIGE_OK;
    auto merge = [&](auto m) { hipLaunchKernelGGL(m, dim3((unsigned)((groups * P + 255) / 256)), dim3(256), 0, st, a); };
    if (P == 1) merge(cache4_merge_kernel<T, 1>);
    else if (P == 4) merge(cache4_merge_kernel<T, 4>);
    else merge(cache4_merge_kernel<T, 16>);
    SIGE_LAUNCH_CHECK("sige_cache4_attn(merge)");
    return SIGE_OK;
}

template <typename T>
static int launch_cache4(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st)
{
    switch ((a.d + 15) / 16) {                     // 16-wide steps over a head
    case 1: return launch_cache4_as<T, 1, true>(a, f, st);
    case 2: return launch_cache4_as<T, 1, false>(a, f, st);
    case 3: return launch_cache4_as<T, 2, true>(a, f, st);
    case 4: return launch_cache4_as<T, 2, false>(a, f, st);
    case 5: return launch_cache4_as<T, 3, true>(a, f, st);
    case 6: return launch_cache4_as<T, 3, false>(a, f, st);
    case 7: return launch_cache4_as<T, 4, true>(a, f, st);
    case 8: return launch_cache4_as<T, 4, false>(a, f, st);
    case 9: return launch_cache4_as<T, 5, true>(a, f, st);
    case 10: return launch_cache4_as<T, 5, false>(a, f, st);
    case 11: return launch_cache4_as<T, 6, true>(a, f, st);
    case 12: return launch_cache4_as<T, 6, false>(a, f, st);
    case 13: return launch_cache4_as<T, 7, true>(a, f, st);
    case 14: return launch_cache4_as<T, 7, false>(a, f, st);
    case 15: return launch_cache4_as<T, 8, true>(a, f, st);
    default: return launch_cache4_as<T, 8, false>(a, f, st);
    }
}

}  // namespace sige
