// sige_cache4_attn, sige_cache4_attn_blocks: checks, the cut of a call into workgroups, dispatch by type (the kernels are in
// cache4_attn.h).
#include "cache4_attn.h"

namespace sige {

// Tokens per chunk, and waves that share the chunks of a workgroup's queries out among them.
static int cache4_chunk(int d, sige_dtype dt, bool common)
{
    const int DT = (d + 31) / 32;
    return 32 * (common ? cache4_common_tiles(DT) : cache4_apart_tiles(DT, dt == SIGE_F32 ? Cache4Compute<float>::parts : 1));
}

// room: floats of workspace, what the splits' partial sums have to fit into.
static Cache4Form plan_cache4(int Nq, int T, int heads, int d, sige_dtype dt, size_t room = ~(size_t)0)
{
    const int DT = (d + 31) / 32;
    const int target = knob(SIGE_KNOB_ATTN_WGS);
    Cache4Form f = {dt != SIGE_F32 && (long)heads * ((Nq + 31) / 32) >= 512, 1};
    const int nk = f.common ? 1 : cache4_apart_waves(DT, dt == SIGE_F32 ? Cache4Compute<float>::parts : 1);
    const long rows = f.common ? 32 * CACHE4_COMMON_WAVES : 32;
    const int KCH = cache4_chunk(d, dt, f.common);
    const long chunks = ((long)T + KCH - 1) / KCH;
    const long base = (long)heads * ((Nq + rows - 1) / rows);
    long want = ((target >= 0 ? target : f.common ? 512 : 256) + base - 1) / base;
    const long cap = chunks / (2 * nk);
    if (want > cap) want = cap;
    if (want > 64) want = 64;
    if (want < 1) want = 1;
    const long per = std::max((chunks + want - 1) / want, 1L);
    f.splits = (int)std::max((chunks + per - 1) / per, 1L);
    while (f.splits > 1 && (size_t)f.splits * heads * Nq * (d + 4) > room) {
        const long fewer = f.splits - 1, p = (chunks + fewer - 1) / fewer;
        f.splits = (int)((chunks + p - 1) / p);
    }
    return f;
}

static int cache4_attn_entry(const char* who, Cache4AttnArgs& a, const void* q, int32_t q_ld, const void* cache, int32_t capacity,
                             sige_dtype dt, int32_t Nq, int32_t T, int32_t heads, int32_t d, float scale, const int32_t* ranges,
                             void* o, int32_t o_ld, void* workspace, size_t workspace_bytes, void* stream)
{
    SIGE_REQUIRE(Nq >= 0 && T >= 0 && heads > 0 && d > 0 && capacity > 0, SIGE_ERR_INVALID_ARG,
                 "%s: need Nq >= 0, T >= 0, heads > 0, d > 0, capacity > 0", who);
    SIGE_REQUIRE(T <= capacity, SIGE_ERR_CAPACITY, "%s: T (%d) exceeds the capacity (%d)", who, T, capacity);
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    const int vw = dt == SIGE_F32 ? 4 : 8;
    SIGE_REQUIRE(d % 8 == 0 && d <= 256, SIGE_ERR_UNSUPPORTED, "%s: d must be a multiple of 8 and <= 256", who);
    SIGE_REQUIRE(heads <= 65535, SIGE_ERR_UNSUPPORTED, "%s: too many heads", who);
    if (Nq == 0) return SIGE_OK;
    SIGE_REQUIRE(q && cache && o, SIGE_ERR_INVALID_ARG, "%s: q, cache and o are required", who);
    SIGE_REQUIRE(q_ld >= (long)heads * d && o_ld >= (long)heads * d, SIGE_ERR_INVALID_ARG, "%s: row strides must be >= heads*d", who);
    SIGE_REQUIRE(q_ld % vw == 0 && o_ld % vw == 0, SIGE_ERR_UNSUPPORTED, "%s: row strides must be multiples of %d elements", who, vw);
    SIGE_REQUIRE(aligned16(q) && aligned16(cache) && aligned16(o), SIGE_ERR_UNSUPPORTED, "%s: pointers must be 16-byte aligned", who);
    SIGE_REQUIRE(scale >= 0.0f, SIGE_ERR_UNSUPPORTED, "%s: the scale must not be negative", who);
    const Cache4Layout l = cache4_layout(d, capacity);
    a.q = q; a.cache = (const uint8_t*)cache; a.o = o; a.ws = (float*)workspace; a.ranges = ranges;
    a.section = l.section; a.cap = l.cap; a.scales = l.scales; a.full = l.full; a.gs_log2 = l.gs_log2;
    a.q_ld = q_ld; a.o_ld = o_ld; a.Nq = Nq; a.T = T; a.heads = heads; a.d = d;
    // (never 0, which would make a number of the -inf of a token out of sight: the smallest float turns every finite logit into 0 too)
    a.scale_log2e = std::max(scale * 1.4426950408889634f, 1.4e-45f);
    a.d_heads = fast_div(heads); a.d_tpb = fast_div(a.q_tpb); a.d_qbw = fast_div(a.q_bw); a.d_dq = fast_div(d / 4);
    const bool room = workspace != nullptr && aligned16(workspace);
    const Cache4Form f = plan_cache4(Nq, T, heads, d, dt, room ? workspace_bytes / sizeof(float) : 0);
    const int KCH = cache4_chunk(d, dt, f.common);
    const int chunks = (int)(((long)T + KCH - 1) / KCH);
    a.splits = f.splits;
    a.chunks_per_split = (chunks + f.splits - 1) / f.splits;
    hipStream_t st = (hipStream_t)stream;
    return dt == SIGE_F32 ? launch_cache4_f32(a, f, st) : dt == SIGE_F16 ? launch_cache4_f16(a, f, st) : launch_cache4_bf16(a, f, st);
}

}  // namespace sige

using namespace sige;

extern "C" size_t sige_cache4_attn_workspace_bytes(int32_t Nq, int32_t T, int32_t heads, int32_t d)
{
    if (Nq <= 0 || T <= 0 || heads <= 0 || d <= 0 || d > 256) return 0;
    const int splits = std::max(plan_cache4(Nq, T, heads, d, SIGE_F16).splits, plan_cache4(Nq, T, heads, d, SIGE_F32).splits);
    return splits <= 1 ? 0 : (size_t)splits * heads * Nq * (d + 4) * sizeof(float);
}

extern "C" int sige_cache4_attn(const void* q, int32_t q_ld, const void* cache, int32_t capacity, sige_dtype dt, int32_t Nq,
                                int32_t T, int32_t heads, int32_t d, float scale, const int32_t* ranges, void* o, int32_t o_ld,
                                void* workspace, size_t workspace_bytes, void* stream)
{
    clear_error();
    Cache4AttnArgs a;
    a.q_blocks = nullptr;
    a.q_tpb = a.q_bw = a.q_H = a.q_W = 1;
    return cache4_attn_entry("sige_cache4_attn", a, q, q_ld, cache, capacity, dt, Nq, T, heads, d, scale, ranges, o, o_ld, workspace,
                             workspace_bytes, stream);
}

extern "C" int sige_cache4_attn_blocks(const void* q, int32_t q_ld, const sige_geom* g, const int32_t* indices, int32_t n_blocks,
                                       const void* cache, int32_t capacity, sige_dtype dt, int32_t T, int32_t heads, int32_t d,
                                       float scale, const int32_t* ranges, void* o, int32_t o_ld, void* workspace,
                                       size_t workspace_bytes, void* stream)
{
    clear_error();
    const char* who = "sige_cache4_attn_blocks";
    if (int rc = check_geom(g, who, nullptr, nullptr)) return rc;
    SIGE_REQUIRE(g->k == 1 && g->stride == 1 && g->pad == 0, SIGE_ERR_UNSUPPORTED,
                 "%s: the geometry must be that of a 1x1, stride-1, unpadded layer", who);
    SIGE_REQUIRE(n_blocks >= 0, SIGE_ERR_INVALID_ARG, "%s: n_blocks must be a host value >= 0", who);
    SIGE_REQUIRE((long)n_blocks * g->block_h * g->block_w <= 0x7fffffffL, SIGE_ERR_UNSUPPORTED, "%s: too many query rows", who);
    SIGE_REQUIRE(n_blocks == 0 || indices != nullptr, SIGE_ERR_INVALID_ARG, "%s: indices are required", who);
    Cache4AttnArgs a;
    a.q_blocks = indices;
    a.q_tpb = g->block_h * g->block_w;
    a.q_bw = g->block_w; a.q_H = g->H_in; a.q_W = g->W_in;
    return cache4_attn_entry(who, a, q, q_ld, cache, capacity, dt, n_blocks * a.q_tpb, T, heads, d, scale, ranges, o, o_ld, workspace,
                             workspace_bytes, stream);
}
