// sige_cache4_attn: attention of the edited query tokens on keys and values held in 4 bits (Sec. 3.2 "Extension to attention
// layers", Fig. "sige-attention": the queries of the edited tokens against all cached keys and values), the kernels.
//
// o_i = sum_t softmax_t(scale q_i . k_t) v_t over the tokens [begin_i, end_i) that the row sees.  As in sige_sparse_attn everything
// runs transposed, so that what belongs to a query stays in one lane (pair): S^T = K Q^T leaves the logits of a query in the
// registers of lanes l and l + 32, and the probabilities feed O^T += V^T P^T straight from there, because the order of the contraction
// is free as long as V^T is read in the same one.
//
// A cached value is exact in bf16 (fp16 queries: in fp16), so a chunk is expanded once per workgroup, on its way from registers
// to LDS: sixteen conversions per 32 channels, the scale folded in by the instruction, against the 32 x 32 logits that every wave
// makes of them.  What differs by type is the other operand: bf16 and fp16 queries enter as they are; a single-precision
// query, and the probabilities beside it, as the sum of three bf16 numbers (24 bits), so that single precision runs on the bf16 matrix
// instructions at a third of their rate (the fp32 ones have a sixteenth) with exact products.
// A probability is rounded to the compute type once (bf16: 2^-9 of each at most, without bias; the values behind it were
// rounded to 2 bits of significand); the denominator adds what was multiplied (a column of ones beside V) where the
// head size leaves a column free, the unrounded values otherwise.
#pragma once

#include "cache4.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace sige {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

struct Cache4AttnArgs {
    const void* q;
    const uint8_t* cache;
    void* o;
    float* ws;                 // partials [split][head][Nq][d + 4]: the d sums, the maximum, the denominator, 2 unused
    const int32_t* ranges;     // [Nq][2]: the tokens a row sees (NULL: all T)
    const int32_t* q_blocks;   // queries by block list, as sige_sparse_attn_blocks
    long section, cap, scales; // of Cache4Layout
    int q_ld, o_ld, Nq, T, heads, d;
    int splits, chunks_per_split;
    int full, gs_log2;
    float scale_log2e;
    int q_tpb, q_bw, q_H, q_W;
    FastDiv d_heads, d_tpb, d_qbw, d_dq;
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

// Two floats as NP pairs of the compute type whose sums they are (to 8 NP bits of bf16).
template <typename C, int NP> __device__ __forceinline__ void split2(float a, float b, uint32_t (&out)[NP])
{
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        out[i] = round2<C>(a, b);
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

#ifndef KTH
#define KTH 3
#define KTF 2
#endif
// 32-key tiles per chunk, by what their logits take in registers
constexpr int cache4_tiles(int DT, int parts) { return DT <= (parts > 1 ? KTF : KTH) ? 2 : 1; }
constexpr int cache4_v_bytes(int DT, int parts) { return 32 * cache4_tiles(DT, parts) * 64 * DT; }      // a chunk's V rows in LDS
// The 64 bytes of group g of a V row: which of the row's groups of 64 bytes holds it.  Four neighbouring keys keep a group on
// different banks, in the writes (a lane per key) and in the transposed reads (four keys per 16 lanes).
template <int DT> __device__ __forceinline__ int cache4_v_group(int key, int g)
{
    return DT % 2 ? g : DT % 4 ? g ^ ((key >> 1) & 1) : g ^ (key & 3);
}

#ifndef WPS
#define WPS(DT, NP) ((NP) > 1 ? 1 : (DT) <= 7 ? 2 : 1)
#endif
// DT = 32-wide tiles over d; ODD: the last one has 16 channels (d % 32 is 8 or 16), and its row 16 is the row of ones.
// Every wave works by itself: 32 queries, K from memory straight into the first product's operands (8 bytes of a key and group per
// lane: the order of the channels is the queries' too), V through the wave's own rows in LDS, which it is transposed out of.  NQ
// waves of a workgroup take different queries, NK the same ones and every NK-th chunk of the tokens; these meet in LDS at the end.
template <typename T, int DT, bool ODD, int NQ, int NK>
__global__ __launch_bounds__(64 * NQ * NK, WPS(DT, Cache4Compute<T>::parts)) void cache4_attend_kernel(Cache4AttnArgs a)
{
    static_assert(NQ == 1 || NK == 1, "queries or keys over the waves");
    using C = typename Cache4Compute<T>::type;
    constexpr int NP = Cache4Compute<T>::parts;
    constexpr unsigned LAST = Cache4Compute<T>::last;
    constexpr int KT = cache4_tiles(DT, NP), KCH = 32 * KT;
    constexpr int VROW = 64 * DT;
    constexpr int DK = 2 * DT - ODD;               // 16-wide steps over d for S^T
    constexpr int VU = KT == 2 ? DT : (DT + 1) / 2;        // groups a lane expands per chunk: of one of 64 keys, or every other one of 32
    constexpr int SW = (DT + 3) / 4;               // words of a token's scales
    constexpr int GS = DT == 1 ? 1 : DT == 2 ? 2 : DT <= 4 ? 4 : 8;
    extern __shared__ uint4 lds4[];
    char* const lds = reinterpret_cast<char*>(lds4);
    const int d = a.d;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wq = NQ > 1 ? wave : 0, wk = NQ > 1 ? 0 : wave;
    const int half = lane >> 5, l32 = lane & 31;
    int qt, head;                                  // (the heads side by side: with eight of them each XCD keeps one in its L2)
    divmod((int)blockIdx.x, a.d_heads, qt, head);
    const int q0 = (qt * NQ + wq) * 32, qi = q0 + l32;
    if (NQ > 1 && q0 >= a.Nq) return;
    const bool q_ok = qi < a.Nq;

    // what the rows see: a row that sees nothing is left out of the bounds and written as zeros
    int begin = 0, end = a.T;
    int lo = 0, hi = a.T, lo_most = 0, hi_least = a.T;
    bool none = a.T == 0;
    if (a.ranges != nullptr) {
        if (q_ok) cache4_range(a.ranges, a.T, qi, begin, end);
        none = !q_ok || begin >= end;
        lo = __builtin_amdgcn_readfirstlane(wave_min(none ? a.T : begin));
        hi = __builtin_amdgcn_readfirstlane(-wave_min(none ? 0 : -end));
        lo_most = __builtin_amdgcn_readfirstlane(-wave_min(none ? 0 : -begin));
        hi_least = __builtin_amdgcn_readfirstlane(wave_min(none ? a.T : end));
    }
    int c = max((int)blockIdx.z * a.chunks_per_split, lo / KCH) + wk;
    const int c_end = min(((int)blockIdx.z + 1) * a.chunks_per_split, (int)(((long)hi + KCH - 1) / KCH));

    char* const vs = lds + wave * cache4_v_bytes(DT, NP);
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
            const int key = min(kt * 32 + l32, last);
#pragma unroll
            for (int g = 0; g < DT; ++g) {
                if (ODD && g == DT - 1) kc[kt][g] = u32x2{*(const uint32_t*)(ksec + a.full * a.cap * 16 + t0 * 8 + (key * 8 + half * 4)), 0u};
                else kc[kt][g] = *(const u32x2*)(ksec + g * a.cap * 16 + t0 * 16 + (key * 16 + half * 8));
            }
            scales(ksec + a.scales + t0 * GS + key * GS, ksc[kt]);
        }
        const int key = min(vkey, last);
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int g = KT == 2 ? u : 2 * u + half;
            if (KT == 1 && 2 * u + 1 >= DT && half) break;          // (an odd number of groups: the last one is the lower half's)
            if (ODD && (KT == 2 ? u == DT - 1 : 2 * u + 1 >= DT - 1 && g == DT - 1)) {
                const u32x2 w = *(const u32x2*)(vsec + a.full * a.cap * 16 + t0 * 8 + key * 8);
                vc[u] = u32x4{w.x, w.y, 0u, 0u};
            } else {
                vc[u] = *(const u32x4*)(vsec + g * a.cap * 16 + t0 * 16 + key * 16);
            }
        }
        scales(vsec + a.scales + t0 * GS + key * GS, vsc);
    };
    // a group's scale; one that is no number is the power of two that the conversion makes NaN of
    auto scale_of = [&](uint32_t word, int shift) {
        const unsigned byte = (word >> shift) & 255u;
        return cache4_scale(byte > LAST ? 255u : byte);
    };
    if (c < c_end) fetch(c);

    // Q fragments (B operand of S^T = K Q^T): the channels that the lane's half of a group of K holds
    u32x4 qf[NP][DK];
    {
        const long qrow = cache4_query_row(a, min(qi, a.Nq - 1));
        const char* const qp = (const char*)a.q + (qrow * a.q_ld + (long)head * d) * (long)sizeof(T);
#pragma unroll
        for (int s = 0; s < DK; ++s) {
            const int dd = ODD && s == DK - 1 ? 16 * s + 8 * half : 32 * (s >> 1) + 16 * half + 8 * (s & 1);
#pragma unroll
            for (int p = 0; p < NP; ++p) qf[p][s] = u32x4{0u, 0u, 0u, 0u};
            if (q_ok && dd < d) {
                if constexpr (sizeof(T) == 4) {
                    float f[8];
                    unpack<float>(*(const uint4*)(qp + dd * 4), f);
                    unpack<float>(*(const uint4*)(qp + dd * 4 + 16), f + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[NP];
                        split2<C, NP>(f[2 * j], f[2 * j + 1], w);
#pragma unroll
                        for (int p = 0; p < NP; ++p) qf[p][s][j] = w[p];
                    }
                } else {
                    qf[0][s] = *(const u32x4*)(qp + dd * 2);
                }
            }
        }
    }
    // V rows: the 16-byte vectors of a group lie in the order of their number ^ ((key >> 2) & 3), for the banks of the writes
    auto v_at = [&](int key, int g, int j) { return key * VROW + cache4_v_group<DT>(key, g) * 64 + ((j ^ ((key >> 2) & 3)) * 16); };
    if constexpr (ODD) {                           // the columns that no group fills (row 16 of the last tile: ones)
        constexpr uint32_t ONE = __is_same(C, f16) ? 0x3c00u : 0x3f80u;
        for (int j = lane; j < KCH * 2; j += 64) *(u32x4*)(vs + v_at(j >> 1, DT - 1, 2 + (j & 1))) = u32x4{j & 1 ? 0u : ONE, 0u, 0u, 0u};
    }
    // where this lane's share of a transposed read starts: four lanes take the 16 columns of one key, four keys per 16 lanes,
    // lane i of the 16 receives column i of the four keys.  (The keys of one lane differ by multiples of 8: one more turn of 2
    // in the order of the vectors for every 8.)
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int rkey = 4 * half + ((lane & 15) >> 2), rvec = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    int r_lo[DT % 2 ? 1 : DT];                     // by tile (an odd number of them: the tiles follow each other)
#pragma unroll
    for (int nt = 0; nt < (DT % 2 ? 1 : DT); ++nt) r_lo[nt] = v_at(rkey, nt, rvec) + (lane & 1) * 8;
    const int r_up = ((rvec ^ half ^ 2) - (rvec ^ half)) * 16;      // what the vector's place differs by 8 keys on

    f32x16 oacc[DT];
#pragma unroll
    for (int nt = 0; nt < DT; ++nt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[nt][r] = 0.0f;
    float m_run = -INFINITY, l_run = 0.0f;

    for (; c < c_end; c += NK) {
        const int t0 = c * KCH;
        // a chunk of which some row does not see everything
        const bool partial = t0 < lo_most || (long)t0 + KCH > hi_least;
        bool lost_v = false;                       // some token's value in it is no number
        if (partial) {
#pragma unroll
            for (int g = 0; g < DT; ++g) lost_v |= ((vsc[g >> 2] >> (8 * (g & 3))) & 255u) > LAST;
            lost_v = __builtin_amdgcn_ballot_w64(lost_v) != 0ull;
        }
        // V rows (LDS operations of a wave stay in order: the last chunk's reads are behind it)
#pragma unroll
        for (int u = 0; u < VU; ++u) {
            const int g = KT == 2 ? u : 2 * u + half;
            const float scale = scale_of(vsc[(KT == 2 ? u : 2 * u) >> 2], KT == 2 ? 8 * (u & 3) : 16 * (u & 1) + 8 * half);
            const bool tail = ODD && (KT == 2 ? u == DT - 1 : 2 * u + 1 >= DT - 1 && g == DT - 1);
            u32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 e = cache4_eight<C>(vc[u][j], scale);
                x[j] = u32x4{e.x, e.y, e.z, e.w};
            }
            // (a value that is no number is left out of a chunk that some row sees only a part of - 0 * NaN is NaN -, and the rows
            // that see it are marked below)
            if (lost_v && __float_as_uint(scale) == 0x7f800000u) {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = u32x4{0u, 0u, 0u, 0u};
            }
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
                const uint4 e = cache4_eight<C>(kc[kt][g][s & 1], scale_of(ksc[kt][g >> 2], 8 * (g & 3)));
#pragma unroll
                for (int p = NP - 1; p >= 0; --p) mma32<C>(u32x4{e.x, e.y, e.z, e.w}, qf[p][s], sacc[kt]);      // (the small parts first)
            }
        if (c + NK < c_end) fetch(c + NK);         // in flight during the softmax and the second product
        // of tile kt this lane holds keys 8 * (r / 4) + 4 * half + r % 4 of its query
        if (partial) {
            unsigned lost = 0;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t0 + kt * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    if (t < begin || t >= end) sacc[kt][r] = -INFINITY;
                    else if (lost_v)
                        for (int g = 0; g < DT; ++g)
                            if (vsec[a.scales + (long)t * GS + g] > LAST) lost |= 1u << g;
                }
            if (lost_v) {
                lost |= (unsigned)__shfl_xor((int)lost, 32);
#pragma unroll
                for (int nt = 0; nt < DT; ++nt)
                    if (lost >> nt & 1u) {
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (!(ODD && nt == DT - 1 && r >= 8)) oacc[nt][r] = NAN;
                    }
            }
        }
        float mr = sacc[0][0];                     // raw logits: the scale (>= 0) goes into the exponent
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mr = fmaxf(mr, sacc[kt][r]);
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mr), __float_as_uint(mr), false, false);
        const float mx = fmaxf(m_run, fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * a.scale_log2e);
        const float m_at = mx == -INFINITY ? 0.0f : mx;             // (only tokens out of sight so far: nothing is subtracted)
        if (__builtin_amdgcn_ballot_w64(mx != m_run) != 0ull) {     // some query's maximum moved
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_at);
            m_run = mx;
            l_run *= alpha;
#pragma unroll
            for (int nt = 0; nt < DT; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[nt][r] *= alpha;
        }
        // (fp16: probabilities times 2^15, numerator and denominator alike, so that those down to 2^-29 keep their 11 bits and
        // only what is below 2^-40 is lost)
        const float m_sub = m_at - (__is_same(C, f16) ? 15.0f : 0.0f);
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sacc[kt][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[kt][r], a.scale_log2e, -m_sub));
        // O^T += V^T P^T, two steps of 16 keys per tile; step s uses registers 8s..8s+7
        float lsum = 0.0f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 pf[NP];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p0 = sacc[kt][8 * s + 2 * j], p1 = sacc[kt][8 * s + 2 * j + 1];
                    uint32_t w[NP];
                    split2<C, NP>(p0, p1, w);
#pragma unroll
                    for (int p = 0; p < NP; ++p) pf[p][j] = w[p];
                    if constexpr (!ODD) lsum += p0 + p1;
                }
#pragma unroll
                for (int nt = 0; nt < DT; ++nt) {
                    char* const at = vs + (kt * 32 + 16 * s) * VROW + (DT % 2 ? r_lo[0] + nt * 64 : r_lo[nt]);
                    union { s16x4 h[2]; u32x4 u; } vf;
                    vf.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(__attribute__((address_space(3))) char*)at);
                    vf.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(__attribute__((address_space(3))) char*)(at + 8 * VROW + r_up));
#pragma unroll
                    for (int p = NP - 1; p >= 0; --p) mma32<C>(vf.u, pf[p], oacc[nt]);
                }
            }
        l_run += lsum;
    }

    float l_tot;
    if constexpr (ODD) l_tot = __shfl(oacc[DT - 1][8], l32);        // row 16 of the last tile: register 8 of the lower half
    else l_tot = l_run + __shfl_xor(l_run, 32);
    if (none) { m_run = -INFINITY; l_tot = 0.0f; }                  // (what such a row added up is not read)
    if constexpr (NQ > 1) {
        if (!q_ok) return;
        const float inv = 1.0f / l_tot;
        float* const w = a.ws + (((long)blockIdx.z * a.heads + head) * a.Nq + qi) * (d + 4);
        if (a.splits > 1 && half == 0) *(float2*)(w + d) = make_float2(m_run, l_tot);
#pragma unroll
        for (int nt = 0; nt < DT; ++nt)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq) {
                const int dd = nt * 32 + 8 * rq + 4 * half;
                if (dd >= d) continue;
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = none ? 0.0f : oacc[nt][4 * rq + e];
                if (a.splits == 1) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = none ? 0.0f : v[e] * inv;
                    T* const out = (T*)a.o + (long)qi * a.o_ld + head * d + dd;
                    if constexpr (sizeof(T) == 4) *(float4*)out = make_float4(v[0], v[1], v[2], v[3]);
                    else *(uint2*)out = make_uint2(round2<T>(v[0], v[1]), round2<T>(v[2], v[3]));
                } else {
                    *(float4*)(w + dd) = make_float4(v[0], v[1], v[2], v[3]);
                }
            }
    } else {
        // the waves' shares of the keys, brought to a common maximum and added in wave order
        float* const comb = reinterpret_cast<float*>(lds);          // [NK][32 queries][d sums, maximum, denominator, 2 unused]
        const int cs = d + 4;
        __syncthreads();                                            // (chunks no longer needed)
        {
            float* const mine = comb + (wk * 32 + l32) * cs;
            if (half == 0) *(float2*)(mine + d) = make_float2(m_run, l_tot);
#pragma unroll
            for (int nt = 0; nt < DT; ++nt)
#pragma unroll
                for (int rq = 0; rq < 4; ++rq) {
                    const int dd = nt * 32 + 8 * rq + 4 * half;
                    if (dd < d)
                        *(float4*)(mine + dd) = none ? make_float4(0.0f, 0.0f, 0.0f, 0.0f)
                                                     : make_float4(oacc[nt][4 * rq], oacc[nt][4 * rq + 1], oacc[nt][4 * rq + 2], oacc[nt][4 * rq + 3]);
                }
        }
        __syncthreads();
        const int dq = d >> 2;
        for (int e = tid; e < 32 * dq; e += 64 * NK) {
            int q, g;
            divmod(e, a.d_dq, q, g);
            const int qq = qt * 32 + q;
            if (qq >= a.Nq) break;
            const float* const src = comb + q * cs;
            float m = -INFINITY, den = 0.0f, num[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < NK; ++w) m = fmaxf(m, src[w * 32 * cs + d]);
#pragma unroll
            for (int w = 0; w < NK; ++w) {
                const float mw = src[w * 32 * cs + d], lw = src[w * 32 * cs + d + 1];
                const float4 v = *(const float4*)(src + w * 32 * cs + 4 * g);
                // (a wave without keys carries -inf, 0 and zeros; one whose values hold a NaN keeps it whatever its weight)
                const float f = mw == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mw - m);
                den += lw * f;
                num[0] += v.x * f; num[1] += v.y * f; num[2] += v.z * f; num[3] += v.w * f;
            }
            if (a.splits == 1) {
                int b, en;
                cache4_range(a.ranges, a.T, qq, b, en);
                const float inv = 1.0f / den;
#pragma unroll
                for (int i = 0; i < 4; ++i) num[i] = b >= en ? 0.0f : num[i] * inv;
                T* const out = (T*)a.o + (long)qq * a.o_ld + head * d + 4 * g;
                if constexpr (sizeof(T) == 4) *(float4*)out = make_float4(num[0], num[1], num[2], num[3]);
                else *(uint2*)out = make_uint2(round2<T>(num[0], num[1]), round2<T>(num[2], num[3]));
            } else {
                float* const w = a.ws + (((long)blockIdx.z * a.heads + head) * a.Nq + qq) * (d + 4);
                *(float4*)(w + 4 * g) = make_float4(num[0], num[1], num[2], num[3]);
                if (g == 0) *(float2*)(w + d) = make_float2(m, den);
            }
        }
    }
}

// The splits' partial results, added in their order: four consecutive channels of a (query, head) per P neighbouring lanes.
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
    T* const out = (T*)a.o + (long)qi * a.o_ld + head * d + dd;
    if constexpr (sizeof(T) == 4) *(float4*)out = make_float4(num[0], num[1], num[2], num[3]);
    else *(uint2*)out = make_uint2(round2<T>(num[0], num[1]), round2<T>(num[2], num[3]));
}

// How a call is cut (cache4.hip) and its launch, one file per type.
struct Cache4Form { int nq, nk, splits; };
int cache4_few_waves(int d, sige_dtype dt);                 // NK of the form whose waves split the keys
int launch_cache4_f32(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st);
int launch_cache4_f16(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st);
int launch_cache4_bf16(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st);

// waves that split the keys: what their chunks and their sums take in LDS, and what a query takes in registers
template <typename T> constexpr int cache4_nk(int DT) { return DT <= (sizeof(T) == 4 ? 2 : 4) ? 8 : 4; }

template <typename T, int DT, bool ODD, int NQ, int NK>
static int launch_cache4_as(const Cache4AttnArgs& a, hipStream_t st)
{
    const size_t rows = (size_t)NQ * NK * cache4_v_bytes(DT, Cache4Compute<T>::parts);
    const size_t lds = NQ > 1 ? rows : std::max(rows, (size_t)NK * 32 * (a.d + 4) * sizeof(float));
    const long tiles = (a.Nq + 32L * NQ - 1) / (32 * NQ) * a.heads;
    SIGE_REQUIRE(tiles < (1L << 31), SIGE_ERR_UNSUPPORTED, "sige_cache4_attn: too many queries");
    auto kern = cache4_attend_kernel<T, DT, ODD, NQ, NK>;
    if (lds > 48 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        SIGE_REQUIRE(e == hipSuccess, SIGE_ERR_HIP, "sige_cache4_attn: cannot reserve %zu bytes of LDS: %s", lds, hipGetErrorString(e));
    }
    hipLaunchKernelGGL(kern, dim3((unsigned)tiles, 1, a.splits), dim3(64 * NQ * NK), lds, st, a);
    SIGE_LAUNCH_CHECK("sige_cache4_attn");
    if (a.splits == 1) return SIGE_OK;
    const long groups = (long)a.Nq * a.heads * (a.d / 4);
    auto merge = [&](auto m, int P) { hipLaunchKernelGGL(m, dim3((unsigned)((groups * P + 255) / 256)), dim3(256), 0, st, a); };
    if (a.splits <= 4) merge(cache4_merge_kernel<T, 1>, 1);
    else if (a.splits <= 16) merge(cache4_merge_kernel<T, 4>, 4);
    else merge(cache4_merge_kernel<T, 16>, 16);             // at most 64 splits
    SIGE_LAUNCH_CHECK("sige_cache4_attn(merge)");
    return SIGE_OK;
}

template <typename T, int DT>
static int launch_cache4_dt(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st)
{
    const bool odd = ((a.d + 15) / 16) & 1;
    if (f.nq > 1) return odd ? launch_cache4_as<T, DT, true, 4, 1>(a, st) : launch_cache4_as<T, DT, false, 4, 1>(a, st);
    constexpr int NK = cache4_nk<T>(DT);
    return odd ? launch_cache4_as<T, DT, true, 1, NK>(a, st) : launch_cache4_as<T, DT, false, 1, NK>(a, st);
}

template <typename T>
static int launch_cache4(const Cache4AttnArgs& a, const Cache4Form& f, hipStream_t st)
{
    switch ((a.d + 31) / 32) {
    case 1: return launch_cache4_dt<T, 1>(a, f, st);
    case 2: return launch_cache4_dt<T, 2>(a, f, st);
    case 3: return launch_cache4_dt<T, 3>(a, f, st);
    case 4: return launch_cache4_dt<T, 4>(a, f, st);
    case 5: return launch_cache4_dt<T, 5>(a, f, st);
    case 6: return launch_cache4_dt<T, 6>(a, f, st);
    case 7: return launch_cache4_dt<T, 7>(a, f, st);
    default: return launch_cache4_dt<T, 8>(a, f, st);
    }
}

}  // namespace sige
