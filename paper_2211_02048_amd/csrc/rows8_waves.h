// The product of two matrices in 8 bits where tiles alone would leave compute units without work: the waves of a workgroup share the
// input channels of one tile of 32 RT rows x 32 CT output channels, each by itself as in the kernel for few rows (blocks by direct loads into places of its own,
// no barrier), and their sums meet in LDS in a fixed order.  Bound by latency and by what a compute unit gets from L2.  Measured: 333 rows, 1288 -> 648
// 3.9 us by 32 x 32 (by the kernel for few rows 5.3, by tiles of 128 x 64 6.1), 333 rows, 5120 -> 1280 9.8 by 32 x 64 (17.9, 17.8).
#pragma once

#include "rows8_tiles.h"

namespace sige {

template <typename T, int RT, int CT, int NBUF, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void rows8_waves_kernel(Linear8Args a)
{
    constexpr int ROWS = 32 * (RT + CT), BLOCK = ROWS * 128, L = ROWS / 8;                 // of both operands; bytes and direct loads of a block
    constexpr int SETS = (ROWS + 63) / 64, WAVE = NBUF * BLOCK + 2 * SETS * 256;           // LDS of a wave: its blocks, two sets of scale words
    static_assert(RT * CT * 4096 <= NBUF * BLOCK && NBUF <= 4, "the sums fit where the blocks were; a set of words is read before the next but one comes");
    using Tile = Tile8<T, false, RT, CT, NBUF>;
    extern __shared__ __attribute__((aligned(16))) unsigned char waves_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 31, h = lane >> 5;
    const int all_rows = rows8_effective(a.rows);
    const int nx = (a.Cout + 32 * CT - 1) / (32 * CT), my = (all_rows + 32 * RT - 1) / (32 * RT);
    if ((int)blockIdx.x >= nx * my) return;
    int tr, tc;
    tile_place(xcd_run(blockIdx.x, nx * my), nx, my, tr, tc);
    const int row0 = tr * 32 * RT, col0 = tc * 32 * CT;
    const int rows = all_rows - row0 < 32 * RT ? all_rows - row0 : 32 * RT, cols = a.Cout - col0 < 32 * CT ? a.Cout - col0 : 32 * CT;
    unsigned char* mine = waves_lds + wave * WAVE;
    // LDS rows: weights, then tokens (rows that are not there: the last one)
    const auto line = [&](int p) {
        const int c = tile_channel<false>(p), r = p - 32 * CT;
        return p < 32 * CT ? a.w + (long)(col0 + (c < cols ? c : cols - 1)) * a.w_ld : a.x + (long)(row0 + (r < rows ? r : rows - 1)) * a.x_ld;
    };
    const unsigned char* from[L];
#pragma unroll
    for (int i = 0; i < L; ++i) from[i] = line(8 * i + (lane >> 3)) + ((lane & 7) ^ ((4 * (i & 1) + (lane >> 4)) & 7)) * 16;
    const unsigned char* scales[SETS];
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        const int p = 64 * i + lane < ROWS ? 64 * i + lane : ROWS - 1, c = tile_channel<false>(p), r = p - 32 * CT;
        scales[i] = p < 32 * CT ? a.ws + (long)(col0 + (c < cols ? c : cols - 1)) * a.ws_ld : a.xs + (long)(row0 + (r < rows ? r : rows - 1)) * a.xs_ld;
    }
    typedef const __attribute__((address_space(1))) void* global_ptr;
    typedef __attribute__((address_space(3))) void* lds_ptr;
    const int per = (a.blocks + WAVES - 1) / WAVES, first = wave * per, last = first + per < a.blocks ? first + per : a.blocks;
    const auto request = [&](int b, int place) {
        if (b == first || (b & 3) == 0) {
#pragma unroll
            for (int i = 0; i < SETS; ++i)
                __builtin_amdgcn_global_load_lds((global_ptr)(scales[i] + (b & ~3)), (lds_ptr)(mine + NBUF * BLOCK + ((b >> 2 & 1) * SETS + i) * 256), 4, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < L; ++i)
            __builtin_amdgcn_global_load_lds((global_ptr)(from[i] + 128 * (long)b), (lds_ptr)(mine + place * BLOCK + i * 1024), 16, 0, 0);
    };
    f32x16 acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
#pragma unroll
    for (int i = 0; i < NBUF; ++i)
        if (first + i < last) request(first + i, i);
    const int off = m * 128 + ((h ^ (m >> 1)) & 7) * 16;
    int place = 0;
    for (int b = first; b < last; ++b) {
        // (newer requests that may still be on their way: NBUF - 1 blocks)
        constexpr int newer = (NBUF - 1) * L;
        if (b + NBUF <= last) __builtin_amdgcn_s_waitcnt(0x0f70 | ((newer < 63 ? newer : 63) & 15) | ((newer < 63 ? newer : 63) >> 4) << 14);
        else __builtin_amdgcn_s_waitcnt(0x0f70);
        asm volatile("" ::: "memory");
        const unsigned* word = (const unsigned*)(mine + NBUF * BLOCK + (b >> 2 & 1) * SETS * 256) + m;
        unsigned ws[CT], xs[RT];
#pragma unroll
        for (int j = 0; j < CT; ++j) ws[j] = word[32 * j] >> 8 * (b & 3);
#pragma unroll
        for (int i = 0; i < RT; ++i) xs[i] = word[32 * (CT + i)] >> 8 * (b & 3);
        const unsigned char* at = mine + place * BLOCK;
        i32x8 wf[2][CT], xf[2][RT];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int o = off ^ 64 * u;
#pragma unroll
            for (int j = 0; j < CT; ++j) wf[u][j] = both(*(const i32x4*)(at + j * 4096 + o), *(const i32x4*)(at + j * 4096 + (o ^ 32)));
#pragma unroll
            for (int i = 0; i < RT; ++i) xf[u][i] = both(*(const i32x4*)(at + (CT + i) * 4096 + o), *(const i32x4*)(at + (CT + i) * 4096 + (o ^ 32)));
        }
#pragma unroll
        for (int n = 0; n < RT * CT; ++n) Tile::mma(wf[0][n % CT], ws[n % CT], xf[0][n / CT], xs[n / CT], acc[n / CT][n % CT]);
        // the reads are done: the place takes the block NBUF further on
        __builtin_amdgcn_s_waitcnt(0xc07f);
        asm volatile("" ::: "memory");
        if (b + NBUF < last) request(b + NBUF, place);
        place = place + 1 < NBUF ? place + 1 : 0;
#pragma unroll
        for (int n = 0; n < RT * CT; ++n) Tile::mma(wf[1][n % CT], ws[n % CT], xf[1][n / CT], xs[n / CT], acc[n / CT][n % CT]);
    }
    // (the instruction works on all lanes: nothing of it may move into the branches below)
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) {
            asm volatile("" : "+v"(acc[i][j]));
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *(f32x4*)(mine + ((i * CT + j) * 4 + e / 4) * 1024 + lane * 16) = f32x4{acc[i][j][e], acc[i][j][e + 1], acc[i][j][e + 2], acc[i][j][e + 3]};
        }
    __syncthreads();
    constexpr int V = Vec16<T>::N;
#pragma unroll
    for (int u0 = 0; u0 < 2 * RT * CT; u0 += WAVES) {
        const int u = u0 + wave;                             // half v of tile t: 8 channels of a row per lane
        if (u >= 2 * RT * CT) continue;
        const int t = u >> 1, c = t % CT * 32 + 16 * (u & 1) + 8 * h, r = t / CT * 32 + m;
        float f[8];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const unsigned char* at = waves_lds + (t * 4 + 2 * (u & 1) + g) * 1024 + lane * 16;
            f32x4 s = *(const f32x4*)at;
#pragma unroll
            for (int w = 1; w < WAVES; ++w) s += *(const f32x4*)(at + w * WAVE);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * g + e] = s[e];
        }
        if (r >= rows) continue;
#pragma unroll
        for (int w = 0; w < 8; w += V) {
            if (c + w >= cols) continue;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = f[w + e];
            if (a.bias) {
                float g[V];
                load_f32_run<V>(a.bias, col0 + c + w, g);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] += g[e];
            }
            if (a.base) {
                float g[V];
                unpack<T>(*(const uint4*)((const T*)a.base + (long)(row0 + r) * a.base_ld + col0 + c + w), g);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] += g[e];
            }
            *(uint4*)((T*)a.y + (long)(row0 + r) * a.y_ld + col0 + c + w) = pack<T>(v);
        }
    }
}

template <typename T, int RT, int CT, int NBUF, int WAVES>
inline int launch_waves(const char* who, const Linear8Args& a, int rows, hipStream_t st)
{
    constexpr int ROWS = 32 * (RT + CT), LDS = WAVES * (NBUF * ROWS * 128 + 2 * ((ROWS + 63) / 64) * 256);
    const long n = parts_of(a.Cout, 32 * CT) * parts_of(rows, 32 * RT);
    SIGE_REQUIRE(n < (1L << 22), SIGE_ERR_UNSUPPORTED, "%s: too many rows and channels", who);
    const auto kern = rows8_waves_kernel<T, RT, CT, NBUF, WAVES>;
    if (int rc = allow_lds(who, (const void*)kern, LDS)) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)n), dim3(64 * WAVES), LDS, st, a);
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

}  // namespace sige
