// sige_rows8_linear, sige_rows8_linear_gated: products of two matrices in 8 bits on the stacked tokens of the active blocks.
//
// One instruction of the matrix unit, v_mfma_scale_f32_16x16x128_f8f6f4, multiplies 16 weight rows by 16 token rows over a whole block of 128
// channels and applies the two blocks' scales: the sums stay where they are from the first block to the last.  The weights are the
// instruction's first operand, so that a lane holds consecutive output channels of one token.
#include "rows8.h"

namespace sige {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// 32 codes of a lane: channels 16 k .. 16 k + 15 and 64 + 16 k .. of a block, k = lane / 16 (any order serves, as long as both operands have it).
struct Codes32 { uint4 lo, hi; };

__device__ __forceinline__ Codes32 load_codes(const unsigned char* row, int k)
{
    return {*(const uint4*)(row + 16 * k), *(const uint4*)(row + 64 + 16 * k)};
}

// c += 16 weight rows x 16 token rows over a block of 128 channels; the scale words' low bytes count.
template <bool EXACT> struct Step8;
template <> struct Step8<false> {
    static __device__ __forceinline__ void run(const Codes32& a, unsigned sa, const Codes32& b, unsigned sb, f32x4& c)
    {
        const i32x8 u = {(int)a.lo.x, (int)a.lo.y, (int)a.lo.z, (int)a.lo.w, (int)a.hi.x, (int)a.hi.y, (int)a.hi.z, (int)a.hi.w};
        const i32x8 v = {(int)b.lo.x, (int)b.lo.y, (int)b.lo.z, (int)b.lo.w, (int)b.hi.x, (int)b.hi.y, (int)b.hi.z, (int)b.hi.w};
        c = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(u, v, c, 0, 0, 0, (int)sa, 0, (int)sb);
    }
};
template <> struct Step8<true> {
    // codes times scales are bf16 numbers: four instructions of 32 channels
    static __device__ __forceinline__ uint4 expand(unsigned lo, unsigned hi, float scale)
    {
        union { decltype(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(0u, 1.0f, false)) v; unsigned u; } p, q, r, t;
        p.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
        q.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        r.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
        t.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
        return make_uint4(p.u, q.u, r.u, t.u);
    }
    static __device__ __forceinline__ void run(const Codes32& a, unsigned sa, const Codes32& b, unsigned sb, f32x4& c)
    {
        typedef __bf16 v8 __attribute__((ext_vector_type(8)));
        const float fa = scale_value(sa & 255u), fb = scale_value(sb & 255u);
        const auto one = [&](unsigned a0, unsigned a1, unsigned b0, unsigned b1) {
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, expand(a0, a1, fa)), __builtin_bit_cast(v8, expand(b0, b1, fb)), c, 0, 0, 0);
        };
        one(a.lo.x, a.lo.y, b.lo.x, b.lo.y);
        one(a.lo.z, a.lo.w, b.lo.z, b.lo.w);
        one(a.hi.x, a.hi.y, b.hi.x, b.hi.y);
        one(a.hi.z, a.hi.w, b.hi.z, b.hi.w);
    }
};

__device__ __forceinline__ float gate_value(float u, float g, int gate)
{
    return gate == SIGE_GATE_GELU ? u * (0.5f * g * (1.0f + erff(g * 0.70710678118654752f))) : u * g / (1.0f + expf(-g));
}

// 16 rows x 128 output channels per workgroup, 16 channels per wave.
template <typename T, bool GATED>
__global__ __launch_bounds__(512) void rows8_linear_kernel(Linear8Args a)
{
    __shared__ unsigned top[8][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, k = lane >> 4;
    const int rows = rows8_effective(a.rows);
    const int row0 = blockIdx.y * 16, c0 = blockIdx.x * 128 + wave * 16;
    if (row0 >= rows) return;
    const int row = row0 + m < rows ? row0 + m : rows - 1;
    const int ch = c0 + m < a.Cout ? c0 + m : a.Cout - 1;
    const unsigned char* x = a.x + (long)row * a.x_ld;
    const unsigned char* xs = a.xs + (long)row * a.xs_ld;
    const unsigned char* w = a.w + (long)ch * a.w_ld;
    const unsigned char* ws = a.ws + (long)ch * a.ws_ld;
    const long gw = (long)a.Cout * a.w_ld, gs = (long)a.Cout * a.ws_ld;
    f32x4 u = {0, 0, 0, 0}, g = {0, 0, 0, 0};
    for (int b = 0; b < a.blocks; ++b) {
        const Codes32 xc = load_codes(x + 128 * b, k);
        const unsigned sx = xs[b];
        Step8<sizeof(T) == 4>::run(load_codes(w + 128 * b, k), ws[b], xc, sx, u);
        if (GATED) Step8<sizeof(T) == 4>::run(load_codes(w + gw + 128 * b, k), ws[gs + b], xc, sx, g);
    }
    asm volatile("" : "+v"(u), "+v"(g));         // (the instruction works on all lanes: nothing of it may move into the branches below)
    const int c = c0 + 4 * k;                    // the lane's channels c .. c + 3 of token row0 + m
    const bool in = row0 + m < rows;
    if constexpr (!GATED) {
        if (!in || c >= a.Cout) return;
        const T* base = a.base ? (const T*)a.base + (long)row * a.base_ld + c : nullptr;
        T* y = (T*)a.y + (long)row * a.y_ld + c;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v = u[i];
            if (a.bias) v += a.bias[c + i];
            if (base) v += to_f32(base[i]);
            y[i] = from_f32<T>(v);
        }
    } else {
        float v[4];
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool real = c + i < a.Cout;
            const float bu = a.bias && real ? a.bias[c + i] : 0.0f, bg = a.bias && real ? a.bias[a.Cout + c + i] : 0.0f;
            v[i] = real ? gate_value(u[i] + bu, g[i] + bg, a.gate) : 0.0f;
            const unsigned bits = finite_bits(v[i]);
            most = bits > most ? bits : most;
        }
        unsigned o = (unsigned)__shfl_xor((int)most, 16);
        most = o > most ? o : most;
        o = (unsigned)__shfl_xor((int)most, 32);
        most = o > most ? o : most;
        if (k == 0) top[wave][m] = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) most = top[i][m] > most ? top[i][m] : most;
        if (!in) return;
        const int sb = scale_byte(most);
        *(unsigned*)(a.q + (long)row * a.q_ld + c) = codes4(v[0], v[1], v[2], v[3], scale_inverse(sb));
        if (wave == 0 && k == 0) {
            unsigned char* s = a.s + (long)row * a.s_ld;
            s[blockIdx.x] = (unsigned char)sb;
            if (blockIdx.x == gridDim.x - 1)
                for (int b = gridDim.x; b & 3; ++b) s[b] = 0;
        }
    }
}

}  // namespace sige

using namespace sige;

static int linear8_check(const char* who, Linear8Args& a, const void* x, int32_t x_ld, const void* x_scales, int32_t xs_ld, int32_t Cin,
                         const int32_t* count, int32_t rows_per_count, int32_t max_rows, int32_t n_rows, const void* w, int32_t w_ld,
                         const void* w_scales, int32_t ws_ld, int32_t Cout, const float* bias, int* rows)
{
    SIGE_REQUIRE(Cin > 0 && Cout > 0, SIGE_ERR_INVALID_ARG, "%s: need Cin > 0 and Cout > 0", who);
    SIGE_REQUIRE(Cin <= (1 << 28) && Cout <= (1 << 28), SIGE_ERR_UNSUPPORTED, "%s: at most 2^28 channels", who);
    if (int rc = rows8_check(who, count, rows_per_count, max_rows, n_rows, &a.rows, rows)) return rc;
    if (int rc = rows8_check_matrix(who, "x", x, x_ld, x_scales, xs_ld, Cin, *rows > 0)) return rc;
    if (int rc = rows8_check_matrix(who, "w", w, w_ld, w_scales, ws_ld, Cin, *rows > 0)) return rc;
    SIGE_REQUIRE((reinterpret_cast<uintptr_t>(bias) & 3u) == 0, SIGE_ERR_UNSUPPORTED, "%s: bias must be 4-byte aligned", who);
    a.x = (const unsigned char*)x; a.xs = (const unsigned char*)x_scales; a.x_ld = x_ld; a.xs_ld = xs_ld;
    a.w = (const unsigned char*)w; a.ws = (const unsigned char*)w_scales; a.w_ld = w_ld; a.ws_ld = ws_ld;
    a.Cout = Cout; a.bias = bias; a.blocks = (Cin + ROW8_BLOCK - 1) / ROW8_BLOCK;
    return SIGE_OK;
}

extern "C" int sige_rows8_linear(const void* x, int32_t x_ld, const void* x_scales, int32_t xs_ld, int32_t Cin, const int32_t* count,
                                 int32_t rows_per_count, int32_t max_rows, int32_t n_rows, const void* w, int32_t w_ld, const void* w_scales,
                                 int32_t ws_ld, int32_t Cout, const float* bias, const void* base, int32_t base_ld, void* y, sige_dtype dt,
                                 int32_t y_ld, void* stream)
{
    clear_error();
    const char* who = "sige_rows8_linear";
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    Linear8Args a = {};
    int rows;
    if (int rc = linear8_check(who, a, x, x_ld, x_scales, xs_ld, Cin, count, rows_per_count, max_rows, n_rows, w, w_ld, w_scales, ws_ld, Cout, bias, &rows))
        return rc;
    const int vw = (int)(16 / dtype_size(dt));
    SIGE_REQUIRE(y_ld >= Cout && (!base || base_ld >= Cout), SIGE_ERR_INVALID_ARG, "%s: the row strides of y and base must be >= Cout", who);
    SIGE_REQUIRE(Cout % vw == 0 && y_ld % vw == 0 && (!base || base_ld % vw == 0), SIGE_ERR_UNSUPPORTED,
                 "%s: Cout and the row strides of y and base must be multiples of %d", who, vw);
    SIGE_REQUIRE(y != base || !y || y_ld == base_ld, SIGE_ERR_UNSUPPORTED, "%s: y == base needs the same row stride", who);
    if (rows == 0) return SIGE_OK;
    SIGE_REQUIRE(y, SIGE_ERR_INVALID_ARG, "%s: y is required", who);
    SIGE_REQUIRE(aligned16(y) && aligned16(base), SIGE_ERR_UNSUPPORTED, "%s: y and base must be 16-byte aligned", who);
    a.base = base; a.base_ld = base_ld; a.y = y; a.y_ld = y_ld;
    const dim3 grid((Cout + 127) / 128, (rows + 15) / 16);
    SIGE_REQUIRE(grid.y < 65536, SIGE_ERR_UNSUPPORTED, "%s: too many rows", who);
    hipStream_t st = (hipStream_t)stream;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(512), 0, st, a); };
    if (dt == SIGE_F32) go(rows8_linear_kernel<float, false>);
    else if (dt == SIGE_F16) go(rows8_linear_kernel<f16, false>);
    else go(rows8_linear_kernel<bf16, false>);
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

extern "C" int sige_rows8_linear_gated(const void* x, int32_t x_ld, const void* x_scales, int32_t xs_ld, int32_t Cin, const int32_t* count,
                                       int32_t rows_per_count, int32_t max_rows, int32_t n_rows, const void* w, int32_t w_ld,
                                       const void* w_scales, int32_t ws_ld, int32_t Cout, const float* bias, sige_gate gate, void* q,
                                       int32_t q_ld, void* scales, int32_t s_ld, void* stream)
{
    clear_error();
    const char* who = "sige_rows8_linear_gated";
    SIGE_REQUIRE(gate == SIGE_GATE_GELU || gate == SIGE_GATE_SILU, SIGE_ERR_INVALID_ARG, "%s: unknown gate %d", who, (int)gate);
    Linear8Args a = {};
    int rows;
    if (int rc = linear8_check(who, a, x, x_ld, x_scales, xs_ld, Cin, count, rows_per_count, max_rows, n_rows, w, w_ld, w_scales, ws_ld, Cout, bias, &rows))
        return rc;
    SIGE_REQUIRE(Cout % 8 == 0, SIGE_ERR_UNSUPPORTED, "%s: Cout must be a multiple of 8", who);
    if (int rc = rows8_check_matrix(who, "the output", q, q_ld, scales, s_ld, Cout, rows > 0)) return rc;
    SIGE_REQUIRE(rows == 0 || (q != x && scales != x_scales), SIGE_ERR_INVALID_ARG, "%s: the output may not be x", who);
    if (rows == 0) return SIGE_OK;
    a.gate = gate; a.q = (unsigned char*)q; a.q_ld = q_ld; a.s = (unsigned char*)scales; a.s_ld = s_ld;
    const dim3 grid((Cout + 127) / 128, (rows + 15) / 16);
    SIGE_REQUIRE(grid.y < 65536, SIGE_ERR_UNSUPPORTED, "%s: too many rows", who);
    hipLaunchKernelGGL((rows8_linear_kernel<bf16, true>), grid, dim3(512), 0, (hipStream_t)stream, a);
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}
