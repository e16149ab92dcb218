// sige_token_lora: low-rank adapters of many requests (or regions of an image) beside a shared projection, on the stacked tokens of
// the active blocks:   y_r = base_r + alpha_i * up_i (down_i x_r),   i = the adapter of the row's block.
//
// Bound by memory: per row and adapter 2 rank (Cin + Cout) operations against (Cin + 2 Cout) values.  One kernel, no workspace: a
// workgroup takes 16 rows, its four waves share the contraction over Cin (the partial products meet in LDS), then each takes stretches of
// the output channels.  Few rows alone would leave most compute units without work, so the output channels are cut over workgroups too,
// each of which repeats the small first product.  Many narrow rows instead: 16 rows for every wave by itself.  Where the 16 rows have
// several adapters there is one pass for each, of which its own rows keep the result; where runs are short (single tokens of many
// requests) every workgroup of a section of 128 runs first counts them into the order of their adapters and takes up to 16 rows of one
// adapter from there, in any place of the section: no sorted copy, no second launch (32 tokens of 32 adapters of rank 32, 1280 -> 1280:
// 63 -> 8.4 us). Measured: 8192 rows of 1280 -> 1280 in fp16, rank 32, 19.2 us, 3.3 TB/s (the first product, its sums in LDS and the
// second follow each other, and all workgroups are in the same phase; 162 KB of weights per workgroup come from L2); 64 rows of 320 ->
// 960 4.4 us, of which a launch is 3. The middle vector down_i x_r stays in 32 bits; the half types' second product takes it as the sum
// of two halves (the rounded value and the rounded remainder: 16 bits of bf16, 22 of fp16).  fp16 has a power of two per row taken off
// before and put back on the sums, so that neither end of its range is in the way.
#include "common.h"

#include <algorithm>
#include <type_traits>

namespace sige {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct LoraArgs {
    const void* x;
    const void* down;
    const void* up;
    const void* base;
    void* y;
    const float* alpha;
    const int32_t* ids;
    const int32_t* count;
    int Cin, Cout, rank, adapters, x_ld, base_ld, y_ld;
    int rows_per_id, max_rows, n_host;
    int span;                  // stretches of output channels per wave
    int group;                 // runs per workgroup where they are grouped by adapter, else 0
    FastDiv d_per, d_group, d_tiles;
};

template <typename T> struct LoraStep;            // one 16-byte vector per lane and operand: 32 (half types) or 16 channels
template <> struct LoraStep<f16> {
    static __device__ __forceinline__ void run(const uint4& a, const uint4& b, f32x4& c)
    {
        typedef _Float16 v8 __attribute__((ext_vector_type(8)));
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <> struct LoraStep<bf16> {
    static __device__ __forceinline__ void run(const uint4& a, const uint4& b, f32x4& c)
    {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <> struct LoraStep<float> {
    // (lane quarter k of instruction i: channel 4 k + i of the step, in both operands)
    static __device__ __forceinline__ void run(const uint4& a, const uint4& b, f32x4& c)
    {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    }
};

// sum * back + base, rounded once (fp16: eight fused operations that take base as it is, and four conversions)
template <typename T> __device__ __forceinline__ uint4 lora_sum(const f32x4 (&sum)[sizeof(T) == 4 ? 1 : 2], float back, const uint4& base)
{
    if constexpr (sizeof(T) == 4) {
        const f32x4 v = sum[0] + __builtin_bit_cast(f32x4, base);
        return __builtin_bit_cast(uint4, v);
    } else {
        typedef float f32x8 __attribute__((ext_vector_type(8)));
        typedef T v8 __attribute__((ext_vector_type(8)));
        f32x8 v;
        if constexpr (__is_same(T, f16)) {
            const v8 b = __builtin_bit_cast(v8, base);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(sum[e >> 2][e & 3], back, (float)b[e]);
        } else {
            float b[8];
            unpack<T>(base, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = sum[e >> 2][e & 3] + b[e];
        }
        return __builtin_bit_cast(uint4, __builtin_convertvector(v, v8));
    }
}

constexpr int LORA_WAVES = 4;
constexpr int LORA_SECTION = 128;                                 // runs that are grouped by adapter

// ALONE: every wave has 16 rows of its own and shares nothing: no barriers, no sums in LDS.  RT = 16-wide tiles over the rank.  The
// registers are bounded for two workgroups per compute unit.  No load is guarded (a guard is a branch of its own): lanes past the end
// read the last vector or row again, and what they make of it is either multiplied by the zeros behind the rank, or not stored.
template <typename T, int RT, bool ALONE>
__global__ __launch_bounds__(64 * LORA_WAVES, 2) void token_lora_kernel(LoraArgs a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int VW = Vec16<T>::N, KS = 4 * VW;                  // channels per lane and per step
    constexpr int KR = (RT * 16 + KS - 1) / KS;                   // steps over the rank
    constexpr int RED = RT * 16 + 4;                              // floats per row of the partial products
    constexpr int HROW = KR * KS + VW;                            // values per row of the middle vectors
    constexpr int AHEAD = RT <= 2 ? 8 : RT <= 4 ? 6 : 4;          // steps over Cin whose operands are on their way together
    constexpr int TU = F32 ? 1 : 2, CU = 16 * TU;                 // products per stretch of output channels, its channels
    constexpr int BATCH = KR <= 1 ? (F32 ? 4 : 5) : KR <= 2 ? 2 : 1;          // stretches whose operands are on their way together
    constexpr int HBUF = (F32 ? 1 : 2) * 16 * HROW / VW;
    __shared__ float red[ALONE ? 1 : LORA_WAVES][16][RED];
    __shared__ uint4 hall[ALONE ? LORA_WAVES : 1][HBUF];
    __shared__ float hscale[16];                                  // fp16: what the rows' sums are multiplied by at the end
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    uint4* const hbuf = hall[ALONE ? wave : 0];
    T* const hs = reinterpret_cast<T*>(hbuf);                     // [value, remainder][16][HROW]
    const int l16 = lane & 15, quarter = lane >> 4;
    long rows = a.n_host;
    if (a.n_host < 0) {
        rows = (long)(*a.count) * a.rows_per_id;
        if (rows > a.max_rows) rows = a.max_rows;
    }
    // the workgroup's rows: l16 stands for one in every lane, `live` if there is one, else a row that there is
    long row;
    bool live;
    int run, rest;
    if (a.group > 0) {
        int section, tile;
        divmod((int)blockIdx.x, a.d_tiles, section, tile);
        if (ALONE) tile = tile * LORA_WAVES + wave;
        const int run0 = section * LORA_SECTION, per = a.rows_per_id;
        if ((long)run0 * per >= rows) return;
        const int n = (int)min((long)LORA_SECTION, (rows + per - 1) / per - run0);       // runs of the section
        // A run's place: how many have a smaller (adapter, run); P threads share its comparisons.  Every a.group-th run of an adapter
        // starts a workgroup's rows.
        constexpr int P = 64 * LORA_WAVES / LORA_SECTION, SHARE = LORA_SECTION / P;
        __shared__ alignas(16) unsigned keys[LORA_SECTION + 4 * P];                     // (shares 16 bytes more apart: other banks)
        __shared__ unsigned sorted[LORA_SECTION], starts[LORA_SECTION];
        if (tid < LORA_SECTION) {
            unsigned k = ~0u;
            if (tid < n) {
                const int i = a.ids[run0 + tid];
                k = (unsigned)((unsigned)i >= (unsigned)a.adapters ? a.adapters : i) * LORA_SECTION + tid;      // (none: behind the others)
            }
            keys[tid + tid / SHARE * 4] = k;
        }
        __syncthreads();
        const int mine = tid / P, part = tid % P;
        const unsigned key = keys[mine + mine / SHARE * 4], start = key & ~(unsigned)(LORA_SECTION - 1);
        int place = 0, before = 0;                                // smaller keys, and those of smaller adapters
#pragma unroll
        for (int j = 0; j < SHARE; j += 4) {
            const uint4 k = *(const uint4*)(keys + part * (SHARE + 4) + j);
            place += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
            before += (k.x < start) + (k.y < start) + (k.z < start) + (k.w < start);
        }
#pragma unroll
        for (int x = 1; x < P; x <<= 1) { place += __shfl_xor(place, x); before += __shfl_xor(before, x); }
        if (part == 0) {
            int q, r = 1;
            if (mine < n) { divmod(place - before, a.d_group, q, r); sorted[place] = key; }
            starts[mine < n ? place : mine] = r == 0;
        }
        __syncthreads();
        const bool s0 = starts[lane] != 0u, s1 = starts[64 + lane] != 0u;
        const unsigned long b0 = __builtin_amdgcn_ballot_w64(s0), b1 = __builtin_amdgcn_ballot_w64(s1);
        const int n0 = __builtin_popcountl(b0), i0 = __builtin_popcountl(b0 & ((1ul << lane) - 1)), i1 = n0 + __builtin_popcountl(b1 & ((1ul << lane) - 1));
        const unsigned long h0 = __builtin_amdgcn_ballot_w64(s0 && i0 == tile), h1 = __builtin_amdgcn_ballot_w64(s1 && i1 == tile);
        if ((h0 | h1) == 0ul) return;
        const int head = h0 != 0ul ? __builtin_ctzl(h0) : 64 + __builtin_ctzl(h1);
        divmod(l16, a.d_per, run, rest);
        live = run < a.group && head + run < n;
        const unsigned at = sorted[live ? head + run : head];
        live = live && at / LORA_SECTION == sorted[head] / LORA_SECTION;
        run = run0 + (int)(at % LORA_SECTION);
        row = (long)run * per + rest;
        live = live && row < rows;
        if (!live) { run = run0; row = (long)run0 * per; }
    } else {
        const long row0 = ((long)blockIdx.x * (ALONE ? LORA_WAVES : 1) + (ALONE ? wave : 0)) * 16;
        if (row0 >= rows) return;
        live = row0 + l16 < rows;
        row = live ? row0 + l16 : row0;
        divmod((int)row, a.d_per, run, rest);
    }
    int id = a.ids[run];                                          // adapter of row l16
    if (!live || (unsigned)id >= (unsigned)a.adapters) id = -1;
    const T* const xr = (const T*)a.x + row * a.x_ld + VW * quarter;
    if (KR * KS > RT * 16)                                        // (the half types' step of 32 over a rank of 16)
        for (int j = ALONE ? lane : tid; j < HBUF; j += ALONE ? 64 : 64 * LORA_WAVES) hbuf[j] = make_uint4(0, 0, 0, 0);
    if constexpr (ALONE) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");          // (zeros first, then the values)

    const unsigned long all = __builtin_amdgcn_ballot_w64(id >= 0);
    unsigned long todo = all;
    auto next = [&]() {                                           // the next adapter of the 16 rows
        const int cur = __builtin_amdgcn_readlane(id, __builtin_ctzl(todo));
        todo &= ~__builtin_amdgcn_ballot_w64(id == cur);
        return cur;
    };
    const int full = a.Cin / KS, tail = a.Cin - full * KS;        // steps, channels of the last one
    const int share = ALONE ? full : (full + LORA_WAVES - 1) / LORA_WAVES;       // of a wave, one after the other: whole lines of memory
    const int part = ALONE ? 0 : wave;
    float back = 1.0f;
    constexpr float LARGEST = __is_same(T, f16) ? 65504.0f : 0x1.fep127f;
    // the middle vector's values q * 4 ... + 3 of token t, scaled by `down`
    auto keep = [&](int t, int q, const float (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            // (half types: single precision ends above bf16, where the value is the type's largest number and a remainder; an infinity
            // is in the remainder: a difference of two would be NaN)
            const T h = from_f32<T>(F32 ? v[i] : fminf(fmaxf(v[i], -LARGEST), LARGEST));
            hs[t * HROW + 4 * q + i] = h;
            if constexpr (!F32) hs[(16 + t) * HROW + 4 * q + i] = from_f32<T>(v[i] - to_f32(h));
        }
    };
    f32x4 alone[RT];                                              // ALONE: the sums of row l16 with its own adapter
    while (todo != 0) {
        // two adapters per pass, where there are two: of their products a lane keeps its own token's
        const int cur0 = next(), cur1 = todo != 0 ? next() : -1;
        f32x4 own[RT];
        for (int n = 0; n < (cur1 >= 0 ? 2 : 1); ++n) {
            const int cur = n == 0 ? cur0 : cur1;
            const T* dr[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                dr[rt] = (const T*)a.down + ((long)cur * a.rank + min(rt * 16 + l16, a.rank - 1)) * a.Cin + VW * quarter;
            f32x4 acc[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[rt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            auto steps = [&](auto count, int s0) {                // that many of the wave's steps, from s0 on
                constexpr int N = decltype(count)::value;
                uint4 xv[N], dv[N][RT];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    xv[i] = *(const uint4*)(xr + (s0 + i) * KS);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) dv[i][rt] = *(const uint4*)(dr[rt] + (s0 + i) * KS);
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) LoraStep<T>::run(dv[i][rt], xv[i], acc[rt]);      // rows: ranks, columns: tokens
            };
            int s = part * share;
            const int end = min(s + share, full);
            for (; s + AHEAD <= end; s += AHEAD) steps(std::integral_constant<int, AHEAD>(), s);
            for (; s < end; ++s) steps(std::integral_constant<int, 1>(), s);
            if (tail != 0 && (ALONE || wave == LORA_WAVES - 1)) { // the last channels
                const bool in = VW * quarter < tail;
                const int at = full * KS - (in ? 0 : VW * quarter);
                uint4 xv = *(const uint4*)(xr + at);
                if (!in) xv = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    uint4 dv = *(const uint4*)(dr[rt] + at);
                    if (!in) dv = make_uint4(0, 0, 0, 0);
                    LoraStep<T>::run(dv, xv, acc[rt]);
                }
            }
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                if (n == 0 || id == cur) own[rt] = acc[rt];
        }
        if constexpr (ALONE) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                if (id >= 0 && (id == cur0 || id == cur1)) alone[rt] = own[rt];
            continue;
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) *(f32x4*)&red[wave][l16][rt * 16 + 4 * quarter] = own[rt];
        __syncthreads();
        constexpr int LANES = RT <= 1 ? 4 : RT <= 2 ? 8 : RT <= 4 ? 16 : 32;     // of a row: four ranks each
        for (int j = tid; j < 16 * LANES; j += 64 * LORA_WAVES) {        // (whole waves)
            const int t = j / LANES, q = j % LANES;
            const int mine = __shfl(id, t);
            if (mine < 0 || (mine != cur0 && mine != cur1)) continue;
            const bool on = LANES == 4 * RT || q < 4 * RT;
            f32x4 s = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (on) {
                s = *(const f32x4*)&red[0][t][4 * q];
#pragma unroll
                for (int w = 1; w < LORA_WAVES; ++w) s += *(const f32x4*)&red[w][t][4 * q];
            }
            const float alpha = a.alpha != nullptr ? a.alpha[mine] : 1.0f;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = 4 * q + i < a.rank ? alpha * s[i] : 0.0f;
            if constexpr (__is_same(T, f16)) {                    // the row's largest value to 2^14..2^15
                unsigned top = 0u;
#pragma unroll
                for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
                for (int x = 1; x < LANES; x <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, x));
                const int e = min(max((int)(top >> 23), 27), 254);         // (a row of zeros, of infinities)
                const float down = __uint_as_float((unsigned)(127 + 127 + 14 - e) << 23);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] *= down;
                if (q == 0) hscale[t] = __uint_as_float((unsigned)(e - 14) << 23);
            }
            if (!on) continue;
            keep(t, q, v);
        }
        __syncthreads();
    }
    if constexpr (ALONE) {
        const float alpha = a.alpha != nullptr && id >= 0 ? a.alpha[id] : 1.0f;
        float v[RT][4];
        unsigned top = 0u;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[rt][i] = id >= 0 && rt * 16 + 4 * quarter + i < a.rank ? alpha * alone[rt][i] : 0.0f;
                top = max(top, __float_as_uint(v[rt][i]) & 0x7fffffffu);
            }
        if constexpr (__is_same(T, f16)) {                        // (as above; the four quarters hold the row)
            top = max(top, (unsigned)__shfl_xor((int)top, 16));
            top = max(top, (unsigned)__shfl_xor((int)top, 32));
            const int e = min(max((int)(top >> 23), 27), 254);
            const float down = __uint_as_float((unsigned)(127 + 127 + 14 - e) << 23);
            back = __uint_as_float((unsigned)(e - 14) << 23);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[rt][i] *= down;
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) keep(l16, rt * 4 + quarter, v[rt]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // (read as other vectors below; a wave's LDS operations stay in order)
    }

    // y^T = up h^T: rows are output channels, so that a lane holds consecutive ones of one token.  Half types: two products of 16
    // whose rows are dealt out in fours, eight consecutive channels per lane.
    uint4 hv[KR], hl[KR];
#pragma unroll
    for (int s = 0; s < KR; ++s) {
        hv[s] = *(const uint4*)(hs + l16 * HROW + s * KS + VW * quarter);
        if constexpr (!F32) hl[s] = *(const uint4*)(hs + (16 + l16) * HROW + s * KS + VW * quarter);
    }
    if constexpr (__is_same(T, f16) && !ALONE) back = id >= 0 ? hscale[l16] : 1.0f;
    int u0 = (blockIdx.y * (ALONE ? 1 : LORA_WAVES) + part) * a.span;
    const int u_end = min(u0 + a.span, (a.Cout + CU - 1) / CU);
    // A batch of stretches.  SAME: all rows that there are have one adapter; else what each makes is taken over by its own rows, not
    // added as zeros (what another adapter holds may be no number).
    auto batch = [&](auto same) {
        constexpr bool SAME = decltype(same)::value;
        uint4 bv[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            bv[i] = make_uint4(0, 0, 0, 0);
            if (a.base != nullptr) bv[i] = *(const uint4*)((const T*)a.base + row * a.base_ld + min((u0 + i) * CU + 4 * TU * quarter, a.Cout - VW));
        }
        f32x4 sum[BATCH][TU];
        if constexpr (!SAME) {
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int t = 0; t < TU; ++t) sum[i][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        todo = all;
        while (SAME || todo != 0) {
            const int cur = next();
            const T* const up = (const T*)a.up + (long)cur * a.Cout * a.rank;
            uint4 uv[BATCH][KR][TU];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
#pragma unroll
                for (int t = 0; t < TU; ++t) {
                    const T* const ur = up + (long)min((u0 + i) * CU + (F32 ? l16 : (l16 >> 2) * 8 + t * 4 + (l16 & 3)), a.Cout - 1) * a.rank;
#pragma unroll
                    for (int s = 0; s < KR; ++s) uv[i][s][t] = *(const uint4*)(ur + min(s * KS + VW * quarter, a.rank - VW));
                }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                f32x4 acc[TU];
#pragma unroll
                for (int t = 0; t < TU; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s < KR; ++s)
#pragma unroll
                    for (int t = 0; t < TU; ++t) {
                        LoraStep<T>::run(uv[i][s][t], hv[s], acc[t]);
                        if constexpr (!F32) LoraStep<T>::run(uv[i][s][t], hl[s], acc[t]);
                    }
#pragma unroll
                for (int t = 0; t < TU; ++t)
                    if (SAME || id == cur) sum[i][t] = acc[t];
            }
            if (SAME) break;
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int c = (u0 + i) * CU + 4 * TU * quarter;
            if (live && u0 + i < u_end && c < a.Cout) *(uint4*)((T*)a.y + row * a.y_ld + c) = lora_sum<T>(sum[i], back, bv[i]);
        }
    };
    // (single precision keeps to the general form, one of which it needs anyway: 8192 rows of 640 -> 640 16.6 us against 16.5 as one
    // adapter, 4096 of 1280 -> 1280 25.3 against 24.3, the smaller calls within 0.1)
    const int first = __builtin_amdgcn_readlane(id, 0);
    const bool same = !F32 && first >= 0 && __builtin_amdgcn_ballot_w64(live && id != first) == 0ul;
    if (same)
        for (; u0 < u_end; u0 += BATCH) batch(std::true_type());
    else
        for (; u0 < u_end; u0 += BATCH) batch(std::false_type());
}

template <typename T>
static int launch_lora(LoraArgs& a, int rows, hipStream_t st)
{
    const int units = (a.Cout * (int)sizeof(T) + 63) / 64;
    // Short runs of several adapters: grouped, so that a workgroup has one adapter, which costs 1 us and workgroups of fewer rows: runs
    // of up to 5 rows of more than two adapters (2048 rows of 640 -> 640 in runs of 4 9.0 against 11.4 us, of 1 7.8 against 19.5; of 8 8.9
    // against 7.6; 1263 in runs of 3 of two adapters 7.1 against 6.3), and of up to 8 where latency counts (128 rows of 1280 -> 1280 7.9
    // against 9.2); from four runs on
    const int per = a.rows_per_id;
    a.group = per <= (rows <= 512 ? 8 : 5) && rows > 3L * per && a.adapters > 2 && a.adapters < 1 << 24 && rows < 1 << 23 ? 16 / per : 0;
    int tiles = (rows + 15) / 16;
    a.d_tiles = a.d_group = fast_div(1);
    // (of n runs at most this many groups, each of one adapter or none; those that there are not end at once)
    auto groups = [&](int n) { return std::min(n, (int)((n + (long)std::min(a.adapters + 1, n) * (a.group - 1)) / a.group)); };
    if (a.group > 0) {
        const int runs = (int)(((long)rows + per - 1) / per), section = groups(LORA_SECTION);
        tiles = runs / LORA_SECTION * section + groups(runs % LORA_SECTION);
        a.d_tiles = fast_div(section);
        a.d_group = fast_div(a.group);
    }
    // Narrow rows, a tile for every SIMD: each wave by itself (16384 rows of 128 -> 128 10.9 -> 5.9 us, of 320 -> 320 13.8 -> 10.1, single
    // tokens of 8 adapters 20 -> 9.4; 8192 of 320 -> 320 7.2 -> 9.0, 24576 of 640 -> 640 22.9 -> 25.9)
    const bool alone = tiles >= 1024 && (long)(a.Cin + a.Cout) * (long)sizeof(T) <= 1280;
    // Else workgroups per 16 rows: one per compute unit where the rows alone are fewer (two take 8.6 instead of 6.8 us for 1011 rows of
    // 640 -> 648 in single precision, half of one 7.8), a stretch of channels per wave at least
    const int cut = alone ? 1 : std::max(std::min((256 + tiles - 1) / tiles, (units + LORA_WAVES - 1) / LORA_WAVES), 1);
    a.span = alone ? units : (units + cut * LORA_WAVES - 1) / (cut * LORA_WAVES);
    if (alone) {
        auto quarters = [](int n) { return (n + LORA_WAVES - 1) / LORA_WAVES; };
        if (a.group > 0) {
            const int runs = (int)(((long)rows + per - 1) / per), section = quarters(groups(LORA_SECTION));
            tiles = runs / LORA_SECTION * section + quarters(groups(runs % LORA_SECTION));
            a.d_tiles = fast_div(section);
        } else {
            tiles = quarters(tiles);
        }
    }
    const dim3 grid(tiles, cut);
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(64 * LORA_WAVES), 0, st, a); };
    auto by_rank = [&](auto al) {
        constexpr bool A = decltype(al)::value;
        const int rt = (a.rank + 15) / 16;
        if (rt == 1) go(token_lora_kernel<T, 1, A>);
        else if (rt == 2) go(token_lora_kernel<T, 2, A>);
        else if (rt == 3) go(token_lora_kernel<T, 3, A>);
        else if (rt == 4) go(token_lora_kernel<T, 4, A>);
        else if (rt == 5) go(token_lora_kernel<T, 5, A>);
        else if (rt == 6) go(token_lora_kernel<T, 6, A>);
        else go(token_lora_kernel<T, 8, A>);
    };
    if (alone) by_rank(std::true_type());
    else by_rank(std::false_type());
    SIGE_LAUNCH_CHECK("sige_token_lora");
    return SIGE_OK;
}

}  // namespace sige

using namespace sige;

extern "C" int sige_token_lora(const void* x, sige_dtype dt, int32_t Cin, int32_t x_ld, const int32_t* count, int32_t rows_per_id,
                               int32_t max_rows, int32_t n_rows, const void* down, const void* up, int32_t rank,
                               int32_t n_adapters, const float* alpha, const int32_t* ids, const void* base, int32_t base_ld,
                               int32_t Cout, void* y, int32_t y_ld, void* stream)
{
    clear_error();
    const char* who = "sige_token_lora";
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    SIGE_REQUIRE(Cin > 0 && Cout > 0 && rank > 0 && n_adapters > 0 && rows_per_id > 0, SIGE_ERR_INVALID_ARG,
                 "%s: need Cin, Cout, rank, n_adapters and rows_per_id > 0", who);
    SIGE_REQUIRE(max_rows >= 0 && n_rows >= -1 && n_rows <= max_rows, n_rows > max_rows ? SIGE_ERR_CAPACITY : SIGE_ERR_INVALID_ARG,
                 "%s: need 0 <= n_rows <= max_rows (or n_rows = -1)", who);
    SIGE_REQUIRE(n_rows >= 0 || count != nullptr, SIGE_ERR_INVALID_ARG, "%s: count is required when n_rows is -1", who);
    SIGE_REQUIRE(x_ld >= Cin && y_ld >= Cout && (base == nullptr || base_ld >= Cout), SIGE_ERR_INVALID_ARG,
                 "%s: row strides must be >= the channel counts", who);
    const int vw = (int)(16 / dtype_size(dt));
    SIGE_REQUIRE(rank <= 128, SIGE_ERR_UNSUPPORTED, "%s: the rank must be <= 128", who);
    SIGE_REQUIRE(Cin <= 1 << 28 && Cout <= 1 << 28, SIGE_ERR_UNSUPPORTED, "%s: too many channels", who);      // (offsets within a row are ints)
    SIGE_REQUIRE(Cin % vw == 0 && Cout % vw == 0 && rank % vw == 0 && x_ld % vw == 0 && y_ld % vw == 0 && (base == nullptr || base_ld % vw == 0),
                 SIGE_ERR_UNSUPPORTED, "%s: channel counts, rank and row strides must be multiples of %d elements", who, vw);
    const int rows = n_rows >= 0 ? n_rows : max_rows;
    if (rows == 0) return SIGE_OK;
    SIGE_REQUIRE(x && down && up && ids && y, SIGE_ERR_INVALID_ARG, "%s: x, down, up, ids and y are required", who);
    SIGE_REQUIRE(aligned16(x) && aligned16(down) && aligned16(up) && aligned16(base) && aligned16(y), SIGE_ERR_UNSUPPORTED,
                 "%s: pointers must be 16-byte aligned", who);
    SIGE_REQUIRE(x != y, SIGE_ERR_UNSUPPORTED, "%s: y cannot be x", who);
    SIGE_REQUIRE(y != base || y_ld == base_ld, SIGE_ERR_UNSUPPORTED, "%s: y == base needs the same row stride", who);
    SIGE_REQUIRE(rows <= (1 << 28) - 16, SIGE_ERR_UNSUPPORTED, "%s: too many rows", who);        // (16 per workgroup of 256, a launch has 2^32 threads)
    LoraArgs a;
    a.x = x; a.down = down; a.up = up; a.base = base; a.y = y; a.alpha = alpha; a.ids = ids; a.count = count;
    a.Cin = Cin; a.Cout = Cout; a.rank = rank; a.adapters = n_adapters; a.x_ld = x_ld; a.base_ld = base_ld; a.y_ld = y_ld;
    a.rows_per_id = rows_per_id; a.max_rows = max_rows; a.n_host = n_rows; a.d_per = fast_div(rows_per_id);
    hipStream_t st = (hipStream_t)stream;
    return dt == SIGE_F32 ? launch_lora<float>(a, rows, st) : dt == SIGE_F16 ? launch_lora<f16>(a, rows, st) : launch_lora<bf16>(a, rows, st);
}
