// Rows held in 8 bits: codes e4m3 [rows][ld] and one scale byte s = 2^(s - 127) per 128 channels, [rows][s_ld]; what the kernels that
// write and read them share.
#pragma once

#include "common.h"

namespace sige {

constexpr int ROW8_BLOCK = 128;                     // channels of a scale
constexpr int ROW8_CHUNK = 512;                     // channels of a scale word: what a wave of the row kernels takes at once

constexpr long ROW8_MOST_WAVES = (1L << 26) - 4;    // four to a workgroup of 256 threads, of which a launch has fewer than 2^32

inline long row8_ld(long C) { return (C + ROW8_BLOCK - 1) / ROW8_BLOCK * ROW8_BLOCK; }
inline long row8_scale_ld(long C) { return (C + ROW8_CHUNK - 1) / ROW8_CHUNK * 4; }

// Which rows a call has: host value or count * rows_per_count on the device.
struct Rows8 {
    const int32_t* count;
    int rows_per_count, max_rows, n_host;
};

__device__ __forceinline__ int rows8_effective(const Rows8& r)
{
    if (r.n_host >= 0) return r.n_host;
    const long n = (long)(*r.count) * r.rows_per_count;
    return (int)(n < 0 ? 0 : n < r.max_rows ? n : r.max_rows);       // (a count below zero is none: as 32 bits the product could be a large number)
}

// Checks of the rows; launch = the most rows there can be.
inline int rows8_check(const char* who, const int32_t* count, int rows_per_count, int max_rows, int n_rows, Rows8* r, int* launch)
{
    SIGE_REQUIRE(max_rows >= 0 && n_rows >= -1 && n_rows <= max_rows, n_rows > max_rows && max_rows >= 0 ? SIGE_ERR_CAPACITY : SIGE_ERR_INVALID_ARG,
                 "%s: need 0 <= n_rows <= max_rows (or n_rows = -1)", who);
    SIGE_REQUIRE(n_rows >= 0 || (count != nullptr && rows_per_count > 0), SIGE_ERR_INVALID_ARG,
                 "%s: count and rows_per_count are required when n_rows is -1", who);
    r->count = count; r->rows_per_count = rows_per_count; r->max_rows = max_rows; r->n_host = n_rows;
    *launch = n_rows >= 0 ? n_rows : max_rows;
    return SIGE_OK;
}

// Checks of a matrix in 8 bits (pointers are looked at where rows > 0 only).
inline int rows8_check_matrix(const char* who, const char* what, const void* q, int q_ld, const void* s, int s_ld, int C, bool used)
{
    SIGE_REQUIRE(q_ld >= row8_ld(C) && s_ld >= row8_scale_ld(C), SIGE_ERR_INVALID_ARG,
                 "%s: %d channels of %s take rows of %ld codes and %ld scale bytes", who, C, what, row8_ld(C), row8_scale_ld(C));
    SIGE_REQUIRE(q_ld % 16 == 0 && s_ld % 4 == 0, SIGE_ERR_UNSUPPORTED, "%s: row strides of %s must be multiples of 16 codes and 4 scale bytes", who, what);
    if (!used) return SIGE_OK;
    SIGE_REQUIRE(q && s, SIGE_ERR_INVALID_ARG, "%s: codes and scales of %s are required", who, what);
    SIGE_REQUIRE(aligned16(q) && (reinterpret_cast<uintptr_t>(s) & 3u) == 0, SIGE_ERR_UNSUPPORTED,
                 "%s: %s: codes must be 16-byte, scales 4-byte aligned", who, what);
    return SIGE_OK;
}

// ---- device side ---------------------------------------------------------------

// The larger of v and what the lanes 8, 4, 2 and 1 places on (cyclically, within 16 lanes) hold: afterwards the maximum over the 16.
__device__ __forceinline__ unsigned max_over_16(unsigned v)
{
#define SIGE_MAX_ROR(n)                                                                                    \
    {                                                                                                      \
        const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + n, 0xf, 0xf, false);    \
        v = o > v ? o : v;                                                                                 \
    }
    SIGE_MAX_ROR(8) SIGE_MAX_ROR(4) SIGE_MAX_ROR(2) SIGE_MAX_ROR(1)
#undef SIGE_MAX_ROR
    return v;
}

// |x| as its bits if it is finite, 0 otherwise (bits of non-negative floats are in the order of the floats).
__device__ __forceinline__ unsigned finite_bits(float x)
{
    const unsigned b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// Scale byte of a block whose largest finite magnitude has these bits: the smallest s >= 1 with max <= 448 * 2^(s - 127)
// (448 = 1.75 * 2^8).
__device__ __forceinline__ int scale_byte(unsigned top)
{
    const int s = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    return s > 1 ? s : 1;
}

// 2^(127 - s), what the block's values are multiplied by (s in 1..247).
__device__ __forceinline__ float scale_inverse(int s) { return __uint_as_float((unsigned)(254 - s) << 23); }

// 2^(s - 127) of any byte: 255 is NaN, 0 is 2^-127.
__device__ __forceinline__ float scale_value(unsigned s)
{
    return __uint_as_float(s == 255u ? 0x7fc00000u : s == 0u ? 0x00400000u : s << 23);
}

// Four floats, scaled, as e4m3 codes (nearest, ties to even; infinities and NaN become NaN codes).
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

// A wave's share of a chunk of 512 channels in registers: half types one vector of 8 channels per lane (16 lanes are a block),
// single precision two of 4 (32 lanes are a block; vector h holds channels 256 h + 4 lane ...).
template <typename T> struct ChunkShape {
    static constexpr int N = Vec16<T>::N;           // channels per vector
    static constexpr int V = 8 / N;                 // vectors per lane
};

// Quantises a chunk and stores it.  f: the lane's values, 0 where they lie behind C.  q, s: the row's codes and scale word at the chunk;
// left: channels of the row from the chunk's first one on (> 0).  Codes behind C up to the next multiple of 128 become 0, the scale
// bytes of blocks that begin behind C too.
template <typename T>
__device__ __forceinline__ void store_chunk(const float (&f)[ChunkShape<T>::V][ChunkShape<T>::N], int lane, int left, unsigned char* q,
                                            unsigned char* s)
{
    constexpr int V = ChunkShape<T>::V, N = ChunkShape<T>::N;
    unsigned word = 0;
#pragma unroll
    for (int h = 0; h < V; ++h) {
        unsigned top = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const unsigned b = finite_bits(f[h][i]);
            top = b > top ? b : top;
        }
        top = max_over_16(top);
        if constexpr (V == 2) {
            const unsigned o = (unsigned)__shfl_xor((int)top, 16);
            top = o > top ? o : top;
        }
        const int sb = scale_byte(top);
        const float inv = scale_inverse(sb);
        const int c = V == 1 ? 8 * lane : 256 * h + 4 * lane;
        if (c < (left + ROW8_BLOCK - 1) / ROW8_BLOCK * ROW8_BLOCK) {
            if constexpr (V == 1)
                *(uint2*)(q + c) = make_uint2(codes4(f[h][0], f[h][1], f[h][2], f[h][3], inv), codes4(f[h][4], f[h][5], f[h][6], f[h][7], inv));
            else
                *(unsigned*)(q + c) = codes4(f[h][0], f[h][1], f[h][2], f[h][3], inv);
        }
        // the four blocks' bytes to one word: lane 0 stores it
#pragma unroll
        for (int b = 0; b < 4 / V; ++b) {
            const int block = V == 1 ? b : 2 * h + b;
            const int byte = __builtin_amdgcn_readlane(sb, b * 16 * V);
            if (block * ROW8_BLOCK < left) word |= (unsigned)byte << (8 * block);
        }
    }
    if (lane == 0) *(unsigned*)s = word;
}

}  // namespace sige
