// sige_token_rope / sige_token_rope_blocks: rotary positions with several axes (an image's y and x, a video's t, y and x) on the
// stacked tokens of the active blocks, between the projection to queries and keys and the attention.
//
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = 2 pi * position[row][axis_j] * turns_j
// for every pair j of a head.  The product is formed in turns and whole turns are taken off inside a fused multiply-add, whose
// only rounding is that of the fraction left, so that a position of 10^6 costs no accuracy (the frequency is held to 48 bits, in
// two floats).
//
// Bound by memory: 3 operations per value against 4 or 8 bytes.  An angle serves all heads of a row: a thread computes the sines
// of one vector (16 bytes; in the split layout both its ends) and passes through `heads / parts` heads, so that the sines, which
// for half types are two instructions of the hardware each (absolute error below 2^-18, against a rounding by up to 2^-8 or 2^-11;
// single precision takes the library's sincospif), stay behind the loads.
// Measured: 8192 rows of 16 heads of 128 in bf16, three axes, halves, 15.1 us, 4.4 TB/s (a large copy reaches 5.2); 16 rows 3.1 us, which is a launch.
#include "common.h"

#include <cmath>

namespace sige {

struct RopeArgs {
    const void* x;
    void* y;
    const sige_rope_pair* pairs;
    const float* positions;
    const int32_t* indices;
    const int32_t* count;
    int x_ld, y_ld, heads, d, n_pairs, n_axes;
    int rows_per_count, max_rows, n_host;
    int parts, slots;          // threads per row and vector that share the heads; vectors (of W values) per head and thread slot
    float frame;
    FastDiv d_pb, d_bw, d_parts, d_slots;
};

template <typename T, int W> struct alignas(W * sizeof(T)) RopeVec { T v[W]; };

// W values per access.  HALVES: pair j is (j, j + n_pairs), the slots are the runs of W pairs and then the runs of W channels
// behind the rotated ones; otherwise pair j is (2j, 2j + 1) and the slots are the runs of W channels.
template <typename T, int W, bool HALVES>
__global__ __launch_bounds__(256) void token_rope_kernel(RopeArgs a)
{
    constexpr int P = HALVES ? W : W / 2;          // pairs per slot
    using Vec = RopeVec<T, W>;
    const unsigned e = blockIdx.x * 256u + threadIdx.x;
    int rp, slot, row, part;
    divmod((int)e, a.d_slots, rp, slot);
    divmod(rp, a.d_parts, row, part);
    long rows = a.n_host;
    if (a.n_host < 0) {
        rows = (long)(*a.count) * a.rows_per_count;
        if (rows > a.max_rows) rows = a.max_rows;
    }
    if (row >= rows) return;
    const int rot = HALVES ? a.n_pairs / W : 0;    // slots of pairs
    const bool turns = HALVES ? slot < rot : slot * P < a.n_pairs;
    const int lo = HALVES ? (turns ? slot * W : 2 * a.n_pairs + (slot - rot) * W) : slot * W;
    const T* xr = (const T*)a.x + (long)row * a.x_ld + lo;
    T* yr = (T*)a.y + (long)row * a.y_ld + lo;
    if (!turns) {                                  // channels that no pair has
        if (xr == yr) return;
        for (int h = part; h < a.heads; h += a.parts) *(Vec*)(yr + h * a.d) = *(const Vec*)(xr + h * a.d);
        return;
    }
    float pos[3] = {0.0f, 0.0f, 0.0f};             // by block list: (y, x) or (frame, y, x)
    if (a.indices != nullptr) {
        int b, p, py, px;
        divmod(row, a.d_pb, b, p);
        divmod(p, a.d_bw, py, px);
        const float fy = (float)(a.indices[2 * b] + py), fx = (float)(a.indices[2 * b + 1] + px);
        if (a.n_axes == 2) { pos[0] = fy; pos[1] = fx; }
        else { pos[0] = a.frame; pos[1] = fy; pos[2] = fx; }
    }
    float cs[P], sn[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int j = slot * P + i;
        cs[i] = 1.0f; sn[i] = 0.0f;
        if (HALVES || j < a.n_pairs) {
            const float4 t = *(const float4*)(a.pairs + j);
            const int axis = __float_as_int(t.z);
            float p = 0.0f;                        // (an axis that the call has no positions for does not turn)
            if (a.indices != nullptr) p = axis == 0 ? pos[0] : axis == 1 ? pos[1] : axis == 2 ? pos[2] : 0.0f;
            else if ((unsigned)axis < (unsigned)a.n_axes) p = a.positions[(long)row * a.n_axes + axis];
            const float r = fmaf(p, t.x, -rintf(p * t.x)) + p * t.y;
            if constexpr (sizeof(T) == 4) {
                sincospif(2.0f * r, &sn[i], &cs[i]);
            } else {
                sn[i] = __builtin_amdgcn_sinf(r);  // (its argument is in turns)
                cs[i] = __builtin_amdgcn_cosf(r);
            }
        }
    }
    for (int h = part; h < a.heads; h += a.parts) {
        if constexpr (HALVES) {
            const Vec u = *(const Vec*)(xr + h * a.d), v = *(const Vec*)(xr + h * a.d + a.n_pairs);
            Vec p, q;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float f = to_f32(u.v[i]), g = to_f32(v.v[i]);
                p.v[i] = from_f32<T>(f * cs[i] - g * sn[i]);
                q.v[i] = from_f32<T>(f * sn[i] + g * cs[i]);
            }
            *(Vec*)(yr + h * a.d) = p;
            *(Vec*)(yr + h * a.d + a.n_pairs) = q;
        } else {
            const Vec u = *(const Vec*)(xr + h * a.d);
            Vec p;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float f = to_f32(u.v[2 * i]), g = to_f32(u.v[2 * i + 1]);
                // (a vector that holds the last pair and channels behind it: those keep their bits)
                const bool on = slot * P + i < a.n_pairs;
                p.v[2 * i] = on ? from_f32<T>(f * cs[i] - g * sn[i]) : u.v[2 * i];
                p.v[2 * i + 1] = on ? from_f32<T>(f * sn[i] + g * cs[i]) : u.v[2 * i + 1];
            }
            *(Vec*)(yr + h * a.d) = p;
        }
    }
}

static int rope_entry(const char* who, RopeArgs& a, sige_dtype dt, int rows, sige_rope_layout layout, hipStream_t st)
{
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    SIGE_REQUIRE(layout == SIGE_ROPE_ADJACENT || layout == SIGE_ROPE_HALVES, SIGE_ERR_INVALID_ARG, "%s: unknown layout %d", who, (int)layout);
    SIGE_REQUIRE(a.heads > 0 && a.d > 0 && a.n_pairs > 0 && 2L * a.n_pairs <= a.d, SIGE_ERR_INVALID_ARG,
                 "%s: need heads > 0, d > 0 and 0 < 2 * n_pairs <= d", who);
    SIGE_REQUIRE(a.x_ld >= (long)a.heads * a.d && a.y_ld >= (long)a.heads * a.d, SIGE_ERR_INVALID_ARG, "%s: row strides must be >= heads*d", who);
    const int vw = (int)(16 / dtype_size(dt));
    SIGE_REQUIRE(a.d % vw == 0 && a.x_ld % vw == 0 && a.y_ld % vw == 0, SIGE_ERR_UNSUPPORTED,
                 "%s: d and the row strides must be multiples of %d elements", who, vw);
    if (rows == 0) return SIGE_OK;
    SIGE_REQUIRE(a.x && a.y && a.pairs && (a.positions || a.indices), SIGE_ERR_INVALID_ARG, "%s: x, y, the table and the positions are required", who);
    SIGE_REQUIRE(aligned16(a.x) && aligned16(a.y) && aligned16(a.pairs), SIGE_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", who);
    SIGE_REQUIRE(a.x != a.y || a.x_ld == a.y_ld, SIGE_ERR_UNSUPPORTED, "%s: x == y needs the same row stride", who);
    int w = vw;                                    // the split layout: as wide as n_pairs allows
    if (layout == SIGE_ROPE_HALVES)
        while (a.n_pairs % w) w /= 2;
    a.slots = layout == SIGE_ROPE_HALVES ? a.n_pairs / w + (a.d - 2 * a.n_pairs) / w : a.d / w;
    // threads that share a row's heads: enough of them that the chip has about 2000 threads per compute unit
    const long base = (long)rows * a.slots;
    long parts = ((1L << 18) + base - 1) / base;
    if (parts > a.heads) parts = a.heads;
    a.parts = (int)parts;
    a.d_slots = fast_div(a.slots);
    a.d_parts = fast_div(a.parts);
    const long threads = base * parts;
    SIGE_REQUIRE(threads < (1L << 31) - 256, SIGE_ERR_UNSUPPORTED, "%s: too many rows", who);
    const dim3 grid((unsigned)((threads + 255) / 256));
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
    auto half = [&](auto t) {
        using T = decltype(t);
        if (layout == SIGE_ROPE_ADJACENT) go(token_rope_kernel<T, 8, false>);
        else if (w == 8) go(token_rope_kernel<T, 8, true>);
        else if (w == 4) go(token_rope_kernel<T, 4, true>);
        else if (w == 2) go(token_rope_kernel<T, 2, true>);
        else go(token_rope_kernel<T, 1, true>);
    };
    if (dt == SIGE_F16) half(f16());
    else if (dt == SIGE_BF16) half(bf16());
    else if (layout == SIGE_ROPE_ADJACENT) go(token_rope_kernel<float, 4, false>);
    else if (w == 4) go(token_rope_kernel<float, 4, true>);
    else if (w == 2) go(token_rope_kernel<float, 2, true>);
    else go(token_rope_kernel<float, 1, true>);
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

}  // namespace sige

using namespace sige;

extern "C" int sige_rope_pairs(const int32_t* axis_pairs, int32_t n_axes, double theta, sige_rope_pair* pairs)
{
    clear_error();
    const char* who = "sige_rope_pairs";
    SIGE_REQUIRE(axis_pairs && pairs, SIGE_ERR_INVALID_ARG, "%s: axis_pairs and pairs are required", who);
    SIGE_REQUIRE(n_axes > 0 && theta > 0.0 && std::isfinite(theta), SIGE_ERR_INVALID_ARG, "%s: need n_axes > 0 and a finite theta > 0", who);
    for (int axis = 0; axis < n_axes; ++axis)
        SIGE_REQUIRE(axis_pairs[axis] >= 0, SIGE_ERR_INVALID_ARG, "%s: axis %d has a negative number of pairs", who, axis);
    for (int axis = 0; axis < n_axes; ++axis)
        for (int i = 0; i < axis_pairs[axis]; ++i, ++pairs) {
            const double f = std::pow(theta, -(double)i / axis_pairs[axis]) / 6.283185307179586476925;
            pairs->turns = (float)f;
            pairs->rest = (float)(f - (double)pairs->turns);
            pairs->axis = axis;
            pairs->unused = 0;
        }
    return SIGE_OK;
}

extern "C" int sige_token_rope(const void* x, sige_dtype dt, int32_t heads, int32_t d, int32_t x_ld, const int32_t* count,
                               int32_t rows_per_count, int32_t max_rows, int32_t n_rows, const sige_rope_pair* pairs,
                               int32_t n_pairs, sige_rope_layout layout, const float* positions, int32_t n_axes, void* y,
                               int32_t y_ld, void* stream)
{
    clear_error();
    const char* who = "sige_token_rope";
    SIGE_REQUIRE(max_rows >= 0 && n_rows >= -1 && n_rows <= max_rows, n_rows > max_rows ? SIGE_ERR_CAPACITY : SIGE_ERR_INVALID_ARG,
                 "%s: need 0 <= n_rows <= max_rows (or n_rows = -1)", who);
    SIGE_REQUIRE(n_rows >= 0 || (count != nullptr && rows_per_count > 0), SIGE_ERR_INVALID_ARG,
                 "%s: count and rows_per_count are required when n_rows is -1", who);
    SIGE_REQUIRE(n_axes > 0, SIGE_ERR_INVALID_ARG, "%s: need n_axes > 0", who);
    RopeArgs a;
    a.x = x; a.y = y; a.pairs = pairs; a.positions = positions; a.indices = nullptr; a.count = count;
    a.x_ld = x_ld; a.y_ld = y_ld; a.heads = heads; a.d = d; a.n_pairs = n_pairs; a.n_axes = n_axes;
    a.rows_per_count = rows_per_count; a.max_rows = max_rows; a.n_host = n_rows; a.frame = 0.0f;
    a.d_pb = a.d_bw = fast_div(1);
    return rope_entry(who, a, dt, n_rows >= 0 ? n_rows : max_rows, layout, (hipStream_t)stream);
}

extern "C" int sige_token_rope_blocks(const void* x, sige_dtype dt, int32_t heads, int32_t d, int32_t x_ld, const sige_geom* g,
                                      const int32_t* indices, const int32_t* count, int32_t max_blocks, int32_t n_blocks,
                                      const sige_rope_pair* pairs, int32_t n_pairs, sige_rope_layout layout, int32_t n_axes,
                                      float frame, void* y, int32_t y_ld, void* stream)
{
    clear_error();
    const char* who = "sige_token_rope_blocks";
    int nl;
    if (int rc = check_geom(g, who, nullptr, nullptr)) return rc;
    if (int rc = check_blocks(count, max_blocks, n_blocks, who, &nl)) return rc;
    SIGE_REQUIRE(g->k == 1 && g->stride == 1 && g->pad == 0, SIGE_ERR_UNSUPPORTED,
                 "%s: tokens are the pixels of the blocks themselves (k = 1, stride 1, no padding)", who);
    SIGE_REQUIRE(n_axes == 2 || n_axes == 3, SIGE_ERR_INVALID_ARG, "%s: the axes are (y, x) or (frame, y, x)", who);
    SIGE_REQUIRE(nl == 0 || indices != nullptr, SIGE_ERR_INVALID_ARG, "%s: indices are required", who);
    const long pb = (long)g->block_h * g->block_w;
    SIGE_REQUIRE(pb * max_blocks < (1L << 31), SIGE_ERR_UNSUPPORTED, "%s: too many tokens", who);
    RopeArgs a;
    a.x = x; a.y = y; a.pairs = pairs; a.positions = nullptr; a.indices = indices; a.count = count;
    a.x_ld = x_ld; a.y_ld = y_ld; a.heads = heads; a.d = d; a.n_pairs = n_pairs; a.n_axes = n_axes;
    a.rows_per_count = (int)pb; a.max_rows = (int)(pb * max_blocks); a.n_host = n_blocks >= 0 ? (int)(pb * n_blocks) : -1;
    a.frame = frame;
    a.d_pb = fast_div((int)pb); a.d_bw = fast_div(g->block_w);
    return rope_entry(who, a, dt, (int)(pb * nl), layout, (hipStream_t)stream);
}
