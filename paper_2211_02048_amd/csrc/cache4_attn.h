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

// waves per SIMD that the registers are shared among, four waves on common chunks, half types: told so, the compiler keeps the sums of
// heads up to 128 in half of what it takes otherwise (4096 queries of 16384 x 8 of 128 580 -> 367 us, 2048 of 4096 x 160 146 -> 85)
constexpr int cache4_side_by_side(int NQ, size_t size) { return NQ > 1 && size == 2 ? 2 : 1; }
constexpr int cache4_keys(int DT, int NQ) { return NQ > 1 && DT <= 4 ? 64 : 32; }       // per chunk
// bytes between V rows in LDS: an odd multiple of 64, so that the keys of a transposed read fall on different banks; between K rows:
// 16 bytes more than the channels
constexpr int cache4_v_row(int DT) { return 64 * (DT | 1); }
constexpr int cache4_k_row(int DT, int ODD) { return 32 * (2 * DT - ODD) + 16; }
constexpr int cache4_chunk_bytes(int DT, int ODD, int NQ) { return cache4_keys(DT, NQ) * (cache4_v_row(DT) + cache4_k_row(DT, ODD)); }

// DT = 32-wide tiles over d; ODD: the last one has 16 channels (d % 32 is 8 or 16), and its row 16 is the row of ones.
// NQ = 4: four waves, 32 queries each, share their chunks (two buffers in LDS: the next chunk is expanded into one while the
// other is multiplied, one barrier per chunk).  NQ = 1: NK waves have the same 32 queries and take every NK-th chunk each; their (maximum,
// denominator, sums) meet in LDS at the end.
template <typename T, int DT, bool ODD, int NQ, int NK>
__global__ __launch_bounds__(64 * NQ * NK, cache4_side_by_side(NQ, sizeof(T))) void cache4_attend_kernel(Cache4AttnArgs a)
{
    static_assert(NQ == 1 || NK == 1, "queries or keys over the waves");
    using C = typename Cache4Compute<T>::type;
    constexpr int NP = Cache4Compute<T>::parts;
    constexpr unsigned LAST = Cache4Compute<T>::last;
    constexpr int KCH = cache4_keys(DT, NQ), KT = KCH / 32;
    constexpr int VROW = cache4_v_row(DT), KROW = cache4_k_row(DT, ODD), CHUNK = cache4_chunk_bytes(DT, ODD, NQ);
    constexpr int DK = 2 * DT - ODD;               // 16-wide steps over d for S^T
    constexpr int UNITS = KCH == 64 ? 2 * DT : DT; // what a wave expands at a time: 64 groups of 32 channels
    constexpr int NU = (UNITS + NQ - 1) / NQ;
    constexpr int NBUF = NQ > 1 ? 2 : 1;
    extern __shared__ uint4 lds4[];
    __shared__ int bad_chunk[NQ > 1 ? 2 : NK];     // the chunk (+ 1) that left a value that is no number out of a buffer
    __shared__ int ends[NQ][4];
    char* const lds = reinterpret_cast<char*>(lds4);
    const int d = a.d;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wq = NQ > 1 ? wave : 0, wk = NQ > 1 ? 0 : wave;
    const int half = lane >> 5, l32 = lane & 31;
    int qt, head;                                  // (the heads side by side: with eight of them each XCD keeps one in its L2)
    divmod((int)blockIdx.x, a.d_heads, qt, head);
    const int q0 = (qt * NQ + wq) * 32, qi = q0 + l32;
    const bool q_ok = qi < a.Nq;

    // what the rows see: a row that sees nothing is left out of the bounds and written as zeros
    int begin = 0, end = a.T;
    if (q_ok) cache4_range(a.ranges, a.T, qi, begin, end);
    const bool none = !q_ok || begin >= end;
    int lo = none ? a.T : begin, hi = none ? 0 : end, lo_most = none ? 0 : begin, hi_least = none ? a.T : end;
    if (a.ranges != nullptr || a.T == 0) {
        lo = wave_min(lo);
        hi = -wave_min(-hi);
        lo_most = -wave_min(-lo_most);
        hi_least = wave_min(hi_least);
    } else {                                       // (all rows see all tokens; rows past Nq compute what no one reads)
        lo = 0; hi = a.T; lo_most = 0; hi_least = a.T;
    }
    if (tid < (NQ > 1 ? 2 : NK)) bad_chunk[tid] = 0;
    if constexpr (NQ > 1) {
        if (lane == 0) { ends[wq][0] = lo; ends[wq][1] = hi; ends[wq][2] = lo_most; ends[wq][3] = hi_least; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NQ; ++w) {
            lo = min(lo, ends[w][0]);
            hi = max(hi, ends[w][1]);
            lo_most = max(lo_most, ends[w][2]);
            hi_least = min(hi_least, ends[w][3]);
        }
    } else {
        __syncthreads();
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    lo_most = __builtin_amdgcn_readfirstlane(lo_most);
    hi_least = __builtin_amdgcn_readfirstlane(hi_least);
    int c_begin = blockIdx.z * a.chunks_per_split, c_end = c_begin + a.chunks_per_split;
    c_begin = max(c_begin, lo / KCH);
    c_end = min(c_end, (hi + KCH - 1) / KCH);

    char* const kv = lds + (NQ > 1 ? 0 : wk * CHUNK);        // a buffer: the K rows, then the V rows
    const uint8_t* const sec = a.cache + 2L * head * a.section;

    // a unit's 64 groups: of 64 keys (KCH 64; K's units, then V's), or of the keys and the values of 32
    u32x4 code[NU];
    unsigned sbyte[NU];
    auto fetch = [&](int c) {
        const long t0 = (long)c * KCH;
        const int last = (int)min((long)KCH, (long)a.T - t0) - 1;   // keys past the end read the last key's
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = wq + NQ * i;
            if (UNITS % NQ != 0 && u >= UNITS) break;
            const int g = KCH == 64 ? (u >= DT ? u - DT : u) : u;
            const int which = KCH == 64 ? (u >= DT) : half;
            const int key = min(KCH == 64 ? lane : l32, last);
            const uint8_t* const base = sec + (which ? a.section : 0);
            if (ODD && g == DT - 1) {
                const u32x2 w = *(const u32x2*)(base + a.full * a.cap * 16 + t0 * 8 + key * 8);
                code[i] = u32x4{w.x, w.y, 0u, 0u};
            } else {
                code[i] = *(const u32x4*)(base + g * a.cap * 16 + t0 * 16 + key * 16);
            }
            sbyte[i] = base[a.scales + (t0 << a.gs_log2) + ((long)key << a.gs_log2) + g];
        }
    };
    // the expanded unit's row in LDS
    auto stage = [&](int c, int buf) {
        const int t0 = c * KCH;
        const bool partial = t0 < lo_most || t0 + KCH > hi_least;
#pragma unroll
        for (int i = 0; i < NU; ++i) {
            const int u = wq + NQ * i;
            if (UNITS % NQ != 0 && u >= UNITS) break;
            const int g = KCH == 64 ? (u >= DT ? u - DT : u) : u;
            const int which = KCH == 64 ? (u >= DT) : half;
            const int key = KCH == 64 ? lane : l32;
            char* const dst = kv + buf * CHUNK + (which ? KCH * KROW + key * VROW : key * KROW) + g * 64;
            const float scale = cache4_scale(sbyte[i]);
            // V rows lie an odd multiple of 64 bytes apart, four lanes on the banks of one: every four lanes start with another of their
            // group's four vectors (else the writes took 60 of the 110 cycles that LDS was busy per chunk, 4096 queries of 16384 x 128)
            u32x4 w = code[i];
            int turn = 0;
            if (which && !(ODD && g == DT - 1)) {
                turn = (key >> 2) & 3;
                if (turn & 1) w = u32x4{w.y, w.z, w.w, w.x};
                if (turn & 2) w = u32x4{w.z, w.w, w.x, w.y};
            }
            uint4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = cache4_eight<C>(w[j], scale);
            const bool bad = sbyte[i] > LAST;
            if (__builtin_amdgcn_ballot_w64(bad) != 0ull) {
                // a group that is no number: NaN for all who see it.  In a chunk of which some row does not see everything its
                // values are left out instead (0 * NaN is NaN), and the rows that see them are marked below.
                const uint32_t nan = __is_same(C, f16) ? 0x7e007e00u : 0x7fc07fc0u;
                const uint32_t v = which && partial ? 0u : nan;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (bad) x[j] = make_uint4(v, v, v, v);
                if (bad && which && partial) bad_chunk[NQ > 1 ? buf : wk] = c + 1;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!(ODD && g == DT - 1 && j >= 2)) *(u32x4*)(dst + 16 * ((j + turn) & 3)) = u32x4{x[j].x, x[j].y, x[j].z, x[j].w};
        }
    };
    int c = c_begin + wk;
    if (c < c_end) fetch(c);

    // Q fragments (B operand of S^T = K Q^T): 8 consecutive channels of this lane's query
    u32x4 qf[NP][DK];
    {
        const long qrow = cache4_query_row(a, min(qi, a.Nq - 1));
        const char* const qp = (const char*)a.q + (qrow * a.q_ld + (long)head * d) * (long)sizeof(T);
#pragma unroll
        for (int s = 0; s < DK; ++s) {
            const int dd = 16 * s + 8 * half;
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
    // the columns of the V rows that no group fills (row 16 of the last tile: ones)
    if constexpr (ODD) {
        constexpr uint32_t ONE = __is_same(C, f16) ? 0x3c00u : 0x3f80u;
        for (int j = NQ > 1 ? tid : lane; j < NBUF * KCH * 2; j += 64 * NQ) {
            const int buf = j / (KCH * 2), key = (j >> 1) % KCH;
            *(uint4*)(kv + buf * CHUNK + KCH * KROW + key * VROW + (DT - 1) * 64 + 32 + (j & 1) * 16) = make_uint4(j & 1 ? 0u : ONE, 0, 0, 0);
        }
    }
    // where this lane's share of a transposed read starts: four lanes take the 16 columns of one key, four keys per 16 lanes,
    // lane i of the 16 receives column i of the four keys
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int tr = KCH * KROW + (4 * half + ((lane & 15) >> 2)) * VROW + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;

    f32x16 oacc[DT];
#pragma unroll
    for (int nt = 0; nt < DT; ++nt)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[nt][r] = 0.0f;
    float m_run = -INFINITY, l_run = 0.0f;

    auto multiply = [&](int c, int buf) {
        const int t0 = c * KCH;
        const char* const ks = kv + buf * CHUNK;
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
                    if (s0 + s < DK) kf[s] = *(const u32x4*)(ks + (kt * 32 + l32) * KROW + (16 * (s0 + s) + 8 * half) * 2);
#pragma unroll
                for (int p = NP - 1; p >= 0; --p)  // (the small parts first)
#pragma unroll
                    for (int s = 0; s < AT_ONCE; ++s)
                        if (s0 + s < DK) mma32<C>(kf[s], qf[p][s0 + s], sacc[kt]);
                if (AT_ONCE < DK) __builtin_amdgcn_sched_barrier(0);
            }
        }
        // of tile kt this lane holds keys 8 * (r / 4) + 4 * half + r % 4 of its query
        if (t0 < lo_most || t0 + KCH > hi_least) { // a chunk of which some row does not see everything
            unsigned lost = 0;
            const bool look = __builtin_amdgcn_readfirstlane(bad_chunk[NQ > 1 ? buf : wk]) == c + 1;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int t = t0 + kt * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                    if (t < begin || t >= end) sacc[kt][r] = -INFINITY;
                    else if (look)
                        for (int g = 0; g < DT; ++g)
                            if (sec[a.section + a.scales + ((long)t << a.gs_log2) + g] > LAST) lost |= 1u << g;
                }
            if (look) {
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
        mr = fmaxf(mr, __shfl_xor(mr, 32));
        const float mx = fmaxf(m_run, mr * a.scale_log2e);
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
                constexpr int TILES = DT > 6 ? 4 : DT;
#pragma unroll
                for (int n0 = 0; n0 < DT; n0 += TILES) {
                    s16x4 vlo[TILES], vhi[TILES];
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt) {
                        if (n0 + nt >= DT) break;
                        char* const at = (char*)ks + tr + (kt * 32 + 16 * s) * VROW + (n0 + nt) * 64;
                        vlo[nt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(__attribute__((address_space(3))) char*)at);
                        vhi[nt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(__attribute__((address_space(3))) char*)(at + 8 * VROW));
                    }
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt) {
                        if (n0 + nt >= DT) break;
                        union { s16x4 h[2]; u32x4 u; } vf;
                        vf.h[0] = vlo[nt];
                        vf.h[1] = vhi[nt];
#pragma unroll
                        for (int p = NP - 1; p >= 0; --p) mma32<C>(vf.u, pf[p], oacc[n0 + nt]);
                    }
                    if (TILES < DT) __builtin_amdgcn_sched_barrier(0);
                }
            }
        l_run += lsum;
    };

    if constexpr (NQ > 1) {
        if (c < c_end) {
            stage(c, 0);
            if (c + 1 < c_end) fetch(c + 1);
        }
        for (int buf = 0; c < c_end; ++c, buf ^= 1) {
            __syncthreads();                       // this chunk's rows are there, the other buffer's have been read
            if (c + 1 < c_end) {
                stage(c + 1, buf ^ 1);
                if (c + 2 < c_end) fetch(c + 2);
            }
            multiply(c, buf);
        }
    } else {
        for (; c < c_end; c += NK) {
            stage(c, 0);                           // (LDS operations of a wave stay in order: the last chunk's reads are behind it)
            if (c + NK < c_end) fetch(c + NK);
            multiply(c, 0);
        }
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
    const size_t lds = NQ > 1 ? 2 * (size_t)cache4_chunk_bytes(DT, ODD, NQ)
                              : std::max((size_t)NK * cache4_chunk_bytes(DT, ODD, NQ), (size_t)NK * 32 * (a.d + 4) * sizeof(float));
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
