// sige_rows8_linear, sige_rows8_linear_gated: products of two matrices in 8 bits on the stacked tokens of the active blocks; checks, and which
// kernel takes a call.
#include "rows8_forms.h"

#include <cmath>

namespace sige {

// What a form takes, in microseconds, by a model fitted to measured calls (620 calls of 1 to 8192 rows and 16 to 8192 channels, drawn evenly over the
// logarithms, every form of each replayed from a graph with inputs that change; off by 5 to 10 %): start + rounds of workgroups over the chip
// * (tile + block * blocks of 128 channels that a wave goes through).  The few-row kernel's workgroups are small and many: its time goes by the blocks of
// a wave, and by blocks and tiles in all.  The form that the model takes costs 0.8 % more than the fastest of those calls in the mean, 26 % at
// most; on 330 other calls 1.4 % (half types), 0.9 % (single precision) and 0.04 % (gated), 27 of them over 5 %, 22 % at most.
struct Linear8Cost {
    int rows, cols, slots, shares;
    float start, tile, block;
};

static float linear8_cost(const Linear8Cost& c, int rows, int cols, int blocks)
{
    const float units = (float)parts_of(rows, c.rows) * (float)parts_of(cols, c.cols) / COMPUTE_UNITS;
    float rounds = std::ceil(units);
    if (c.slots == 2) rounds = units <= 1.0f ? 0.62f : units <= 2.0f ? 1.0f : units / 2.0f;     // (one workgroup by itself has the compute unit's time)
    if (c.rows == 256) {
        const float whole = std::floor(units), over = units - whole;
        rounds = whole + (over == 0.0f ? 0.0f : whole >= 1.0f && over <= 0.5f ? 0.62f : 1.0f);  // (the rest as halves)
    }
    return c.start + rounds * (c.tile + c.block * (float)((blocks + c.shares - 1) / c.shares));
}

static float linear8_few_cost(bool exact, int rows, int cols, int blocks)
{
    const int words = (blocks + 3) / 4, waves = words < 8 ? words : 8;
    const float units = (float)parts_of(rows, 16) * (float)parts_of(cols, 16) / COMPUTE_UNITS, steps = (float)(4 * ((words + waves - 1) / waves));
    return exact ? 1.23f + 0.435f * steps + 0.064f * units * (float)blocks + 0.105f * units
                 : 1.54f + 0.315f * steps + 0.066f * units * (float)blocks + 0.027f * units;
}

// The form with the smallest cost that can take the call: the kernels for tiles have 32-bit offsets into a tile's rows.
static int linear8_form(const Linear8Args& a, int rows, bool exact)
{
    static const Linear8Cost half[LINEAR8_FORMS] = {{}, {32, 32, 1, 4, 1.28f, 1.49f, 0.347f}, {32, 64, 1, 4, 0.99f, 1.87f, 0.523f}, {64, 64, 1, 4, 0.48f, 2.75f, 0.726f},
                                                   {128, 64, 2, 1, 0.63f, 3.50f, 0.553f}, {128, 128, 2, 1, 0.0f, 5.17f, 0.838f}, {128, 128, 1, 1, 0.57f, 3.32f, 0.444f},
                                                   {256, 256, 1, 1, 0.0f, 8.73f, 1.057f}};
    static const Linear8Cost single[LINEAR8_FORMS] = {{}, {32, 32, 1, 4, 1.16f, 1.71f, 0.509f}, {32, 64, 1, 4, 0.93f, 2.10f, 0.737f}, {64, 64, 1, 4, 0.0f, 3.47f, 1.080f},
                                                     {128, 64, 2, 1, 0.0f, 4.89f, 0.970f}, {128, 128, 2, 1, 0.0f, 6.13f, 1.397f}, {128, 128, 1, 1, 0.0f, 4.57f, 0.880f}, {}};
    const int set = knob(SIGE_KNOB_ROWS8_FORM);
    const bool offsets = a.x_ld < (1 << 22) && a.w_ld < (1 << 22);
    if (set >= 0 && (set < LINEAR8_TILE_128X64 || offsets)) return set;
    int best = LINEAR8_FEW;
    float least = rows <= 65535 * 16 ? linear8_few_cost(exact, rows, a.Cout, a.blocks) : INFINITY;
    for (int f = LINEAR8_WAVES_32; f < (exact ? LINEAR8_TILE_256 : LINEAR8_FORMS); ++f) {
        if (f >= LINEAR8_TILE_128X64 && !offsets) break;
        const float c = linear8_cost(exact ? single[f] : half[f], rows, a.Cout, a.blocks);
        if (c < least) { least = c; best = f; }
    }
    return best;
}

static int linear8_gated_form(const Linear8Args& a, int rows)
{
    static const Linear8Cost cost[GATED8_FORMS] = {{16, 128, 1, 1, 0.84f, 2.91f, 0.374f}, {64, 128, 1, 1, 1.68f, 3.61f, 0.457f}, {128, 128, 1, 1, 1.22f, 6.22f, 0.653f},
                                                  {256, 128, 1, 1, 0.0f, 11.55f, 1.034f}};
    const int set = knob(SIGE_KNOB_ROWS8_FORM);
    const bool offsets = a.x_ld < (1 << 22) && a.w_ld < (1 << 22);
    if (set >= 0 && (set < GATED8_TILE_64 || offsets)) return set;
    int best = GATED8_FEW;
    float least = INFINITY;
    for (int f = GATED8_FEW; f < (offsets ? GATED8_FORMS : GATED8_TILE_64); ++f) {
        const float c = linear8_cost(cost[f], rows, a.Cout, a.blocks);
        if (c < least) { least = c; best = f; }
    }
    return best;
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
    // (workgroups write while others still read: the base is read by the lane that writes it)
    for (const void* p : {x, x_scales, w, w_scales, (const void*)bias})
        SIGE_REQUIRE(y != p, SIGE_ERR_INVALID_ARG, "%s: y in the place of x, w, their scales or the bias", who);
    a.base = base; a.base_ld = base_ld; a.y = y; a.y_ld = y_ld;
    hipStream_t st = (hipStream_t)stream;
    const int form = linear8_form(a, rows, dt == SIGE_F32);
    return dt == SIGE_F32 ? linear8_f32(who, a, rows, form, st) : dt == SIGE_F16 ? linear8_f16(who, a, rows, form, st) : linear8_bf16(who, a, rows, form, st);
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
    if (rows == 0) return SIGE_OK;
    const int form = linear8_gated_form(a, rows);
    SIGE_REQUIRE(form < GATED8_FORMS, SIGE_ERR_UNSUPPORTED, "%s: the call has no form %d", who, form);
    for (const void* p : {x, x_scales, w, w_scales, (const void*)bias})
        SIGE_REQUIRE(q != p && scales != p, SIGE_ERR_INVALID_ARG, "%s: codes or scales in the place of x, w, their scales or the bias", who);
    SIGE_REQUIRE(q != scales, SIGE_ERR_INVALID_ARG, "%s: codes and scales in one place", who);
    a.gate = gate; a.q = (unsigned char*)q; a.q_ld = q_ld; a.s = (unsigned char*)scales; a.s_ld = s_ld;
    return linear8_gated(who, a, rows, form, (hipStream_t)stream);
}
