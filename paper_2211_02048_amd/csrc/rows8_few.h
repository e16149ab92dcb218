// The product of two matrices in 8 bits for few rows: bound by the way of the weights from memory, and by latency where there are few of
// them.
//
// A wave has 16 CT output channels and 16 RT rows (v_mfma_scale_f32_16x16x128_f8f6f4: a whole block of 128 channels per instruction) and works by
// itself: blocks come by direct loads, whole 128-byte lines, into places in LDS of its own, NBUF of them on their way at a time, and from there
// into the operands; no barrier.  (Loaded straight into the operands, a request has halves of 16 lines: 82 KB per workgroup on 80
// compute units took 3.5 us, whole lines 2.1, of which a launch is 1.9.)  Plain: the waves of a workgroup share the input channels, 512 at a time (a
// scale word), and their sums meet in LDS in a fixed order.  Gated: eight waves side by side have the 128 output channels of
// a block, values and gates of 16 each, so that the row's scale is a maximum over the workgroup.  Measured: 16 rows, 5120 -> 1280 4.1 us, 1280 ->
// 2 x 5120 gated 8.0 (40 workgroups of 330 KB each).
#pragma once

#include "rows8_linear.h"

namespace sige {

// 16 weight rows x 16 token rows over a block of 128 channels; the scale words' low bytes count.
template <bool EXACT>
__device__ __forceinline__ void few_step(const i32x8& w, unsigned ws, const i32x8& x, unsigned xs, f32x4& c)
{
    if constexpr (!EXACT) {
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, c, 0, 0, 0, (int)ws, 0, (int)xs);
    } else {
        const float fw = scale_value(ws & 255u), fx = scale_value(xs & 255u);
#pragma unroll
        for (int i = 0; i < 8; i += 2)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(expand8(w[i], w[i + 1], fw), expand8(x[i], x[i + 1], fx), c, 0, 0, 0);
    }
}

template <bool GATED, int RT, int CT, int NBUF>
struct Few8 {
    static constexpr int BLOCK = (RT + CT) * 2048, L = 2 * (RT + CT);       // bytes and direct loads of a block
    static constexpr int WAVE = NBUF * BLOCK + 512;                         // LDS of a wave: its blocks, two sets of scale words
    static_assert(RT + CT <= 4 && RT * CT * 1024 <= WAVE, "a scale word per lane; the sums fit where the blocks were");
};

template <typename T, bool GATED, int RT, int CT, int NBUF>
__global__ __launch_bounds__(512) void rows8_few_kernel(Linear8Args a)
{
    using S = Few8<GATED, RT, CT, NBUF>;
    constexpr bool EXACT = sizeof(T) == 4;
    static_assert(!GATED || (CT == 2 && NBUF >= 2), "values and gates");
    extern __shared__ __attribute__((aligned(16))) unsigned char few_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, k = lane >> 4;
    const int waves = GATED ? 1 : blockDim.x >> 6;           // that share the input channels
    const int rows = rows8_effective(a.rows);
    const int row0 = blockIdx.y * 16 * RT, c0 = GATED ? blockIdx.x * 128 + wave * 16 : blockIdx.x * 16 * CT;
    if (row0 >= rows) return;
    unsigned char* mine = few_lds + wave * S::WAVE;
    // direct loads: 8 rows of 128 bytes at a time, lane l piece (l % 8) ^ (row / 2 % 8) of row l / 8; rows that are not there: the last one
    const auto weight_row = [&](int t, int r) {
        const int c = c0 + (GATED ? 0 : 16 * t) + r;
        return (long)(c < a.Cout ? c : a.Cout - 1) + (GATED && t ? (long)a.Cout : 0L);
    };
    const auto token_row = [&](int t, int r) { return (long)(row0 + 16 * t + r < rows ? row0 + 16 * t + r : rows - 1); };
    const unsigned char* from[2 * (RT + CT)];
#pragma unroll
    for (int i = 0; i < 2 * (RT + CT); ++i) {
        const int r = 8 * (i & 1) + (lane >> 3), piece = ((lane & 7) ^ (r >> 1)) * 16, t = i >> 1;
        from[i] = (t < CT ? a.w + weight_row(t, r) * a.w_ld : a.x + token_row(t - CT, r) * a.x_ld) + piece;
    }
    // lanes 16 t + r: the scale word of row r of tile t
    const int st = k < RT + CT ? k : RT + CT - 1;
    const unsigned char* scales = st < CT ? a.ws + weight_row(st, m) * a.ws_ld : a.xs + token_row(st - CT, m) * a.xs_ld;
    typedef const __attribute__((address_space(1))) void* global_ptr;
    typedef __attribute__((address_space(3))) void* lds_ptr;

    const int words = (a.blocks + 3) / 4, first = GATED ? 0 : wave, passes = first < words ? (words - first + waves - 1) / waves : 0, n = 4 * passes;
    const auto request = [&](int idx, int place) {           // the wave's block idx (behind the last: the last once more)
        const int word = first + waves * (idx >> 2), want = 4 * word + (idx & 3), b = want < a.blocks ? want : a.blocks - 1;
        if ((idx & 3) == 0) __builtin_amdgcn_global_load_lds((global_ptr)(scales + 4 * (long)word), (lds_ptr)(mine + NBUF * S::BLOCK + (idx >> 2 & 1) * 256), 4, 0, 0);
#pragma unroll
        for (int i = 0; i < S::L; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(from[i] + 128 * (long)b), (lds_ptr)(mine + place * S::BLOCK + i * 1024), 16, 0, 0);
    };
    f32x4 acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < NBUF; ++i)
        if (i < n) request(i, i);
    const int off = m * 128 + ((k ^ (m >> 1)) & 7) * 16;
    int place = 0;
    for (int p = 0; p < passes; ++p) {
        const int word = first + waves * p;
        unsigned ws[CT], xs[RT];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int idx = 4 * p + e;
            // newer requests that may still be on their way: NBUF - 1 blocks, and the scale word that comes with every fourth
            constexpr int all = (NBUF - 1) * S::L;
            const bool with_word = e + NBUF - 1 >= 4;
            if (idx + NBUF - 1 >= n) __builtin_amdgcn_s_waitcnt(0x0f70);
            else if (with_word) __builtin_amdgcn_s_waitcnt(0x0f70 | ((all + 1) & 15) | ((all + 1) >> 4) << 14);
            else __builtin_amdgcn_s_waitcnt(0x0f70 | (all & 15) | (all >> 4) << 14);
            asm volatile("" ::: "memory");
            if (e == 0) {
                const unsigned* w = (const unsigned*)(mine + NBUF * S::BLOCK + (p & 1) * 256);
#pragma unroll
                for (int j = 0; j < CT; ++j) ws[j] = w[16 * j + m];
#pragma unroll
                for (int i = 0; i < RT; ++i) xs[i] = w[16 * (CT + i) + m];
            }
            if (4 * word + e < a.blocks) {
                const unsigned char* at = mine + place * S::BLOCK;
                i32x8 xf[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) xf[i] = both(*(const i32x4*)(at + (CT + i) * 2048 + off), *(const i32x4*)(at + (CT + i) * 2048 + (off ^ 64)));
#pragma unroll
                for (int j = 0; j < CT; ++j) {
                    const i32x8 wf = both(*(const i32x4*)(at + j * 2048 + off), *(const i32x4*)(at + j * 2048 + (off ^ 64)));
#pragma unroll
                    for (int i = 0; i < RT; ++i) few_step<EXACT>(wf, ws[j] >> 8 * e, xf[i], xs[i] >> 8 * e, acc[i][j]);
                }
                // (the instruction works on all lanes: nothing of it may move into the branches below; nor may the reads of this place
                // move behind what is requested into it)
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int j = 0; j < CT; ++j) asm volatile("" : "+v"(acc[i][j]) :: "memory");
            }
            if (idx + NBUF < n) {
                __builtin_amdgcn_s_waitcnt(0xc07f);          // lgkmcnt(0): the reads are done
                asm volatile("" ::: "memory");
                request(idx + NBUF, place);
            }
            place = place + 1 < NBUF ? place + 1 : 0;
        }
    }
    if constexpr (!GATED) {
        if (waves > 1) {
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < CT; ++j) *(f32x4*)(mine + (i * CT + j) * 1024 + lane * 16) = acc[i][j];
            __syncthreads();
        }
        // tile t's sums to wave t % waves: channels c ... c + 3 of a row per lane
#pragma unroll
        for (int t = 0; t < RT * CT; ++t) {
            if (t % waves != wave) continue;
            f32x4 v = acc[t / CT][t % CT];
            if (waves > 1) {
                v = *(const f32x4*)(few_lds + t * 1024 + lane * 16);
                for (int w = 1; w < waves; ++w) v += *(const f32x4*)(few_lds + w * S::WAVE + t * 1024 + lane * 16);
            }
            const int r = row0 + t / CT * 16 + m, c = c0 + t % CT * 16 + 4 * k;
            if (r >= rows || c >= a.Cout) continue;
            if (a.bias) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += a.bias[c + e];
            }
            typedef T t4 __attribute__((ext_vector_type(4)));
            if (a.base) {
                const t4 g = *(const t4*)((const T*)a.base + (long)r * a.base_ld + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += to_f32(g[e]);
            }
            t4 o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = from_f32<T>(v[e]);
            *(t4*)((T*)a.y + (long)r * a.y_ld + c) = o;
        }
    } else {
        unsigned* top = (unsigned*)few_lds;                  // [8][16 RT]
        const int c = c0 + 4 * k;
        const bool real = c < a.Cout;                        // (Cout is a multiple of 8)
        float bu[4] = {0, 0, 0, 0}, bg[4] = {0, 0, 0, 0};
        if (a.bias && real) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { bu[e] = a.bias[c + e]; bg[e] = a.bias[a.Cout + c + e]; }
        }
        float most[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            most[i] = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float u = real ? acc[i][0][e] + bu[e] : 0.0f, g = real ? acc[i][1][e] + bg[e] : 0.0f;
                acc[i][0][e] = a.gate == SIGE_GATE_GELU ? gate_value<SIGE_GATE_GELU>(u, g) : gate_value<SIGE_GATE_SILU>(u, g);
                most[i] = fmaxf(most[i], finite_or_0(acc[i][0][e]));
            }
            most[i] = fmaxf(most[i], __shfl_xor(most[i], 16));
            most[i] = fmaxf(most[i], __shfl_xor(most[i], 32));
        }
        __syncthreads();                                     // (every wave has read its blocks)
#pragma unroll
        for (int i = 0; i < RT; ++i)
            if (k == 0) top[wave * 16 * RT + 16 * i + m] = __float_as_uint(most[i]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = row0 + 16 * i + m;
            unsigned max = 0;
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                const unsigned o = top[w * 16 * RT + 16 * i + m];
                max = o > max ? o : max;
            }
            if (r >= rows) continue;
            const int sb = scale_byte(max);
            *(unsigned*)(a.q + (long)r * a.q_ld + c) = codes4(acc[i][0][0], acc[i][0][1], acc[i][0][2], acc[i][0][3], scale_inverse(sb));
            if (wave == 0 && k == 0) {
                unsigned char* s = a.s + (long)r * a.s_ld;
                s[blockIdx.x] = (unsigned char)sb;
                if (blockIdx.x == gridDim.x - 1)
                    for (int b = gridDim.x; b & 3; ++b) s[b] = 0;
            }
        }
    }
}

template <typename T, bool GATED, int RT, int CT, int NBUF>
inline int launch_few(const char* who, const Linear8Args& a, int rows, int most_waves, hipStream_t st)
{
    using S = Few8<GATED, RT, CT, NBUF>;
    const long nx = parts_of(a.Cout, GATED ? 128 : 16 * CT), my = parts_of(rows, 16 * RT);
    SIGE_REQUIRE(my < 65536 && nx < (1L << 23), SIGE_ERR_UNSUPPORTED, "%s: too many rows or channels", who);
    const dim3 grid((unsigned)nx, (unsigned)my);
    const auto kern = rows8_few_kernel<T, GATED, RT, CT, NBUF>;
    const int words = (a.blocks + 3) / 4, waves = GATED ? 8 : words < most_waves ? words : most_waves;
    if (int rc = allow_lds(who, (const void*)kern, waves * S::WAVE)) return rc;
    hipLaunchKernelGGL(kern, grid, dim3(waves * 64), waves * S::WAVE, st, a);
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

}  // namespace sige
