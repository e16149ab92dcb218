// sige_cache4_attn, sige_cache4_attn_blocks: checks, the cut of a call into workgroups, dispatch by type (the kernels are in
// cache4_attn.h).
#include "cache4_attn.h"

namespace sige {

// How the queries and tokens of a call are dealt out, by its form: queries per workgroup, waves that share its tokens, tokens per chunk.
struct Cache4Cut { int rows, waves, chunk; };
static Cache4Cut cache4_cut(int d, sige_dtype dt, bool many)
{
    const int DT = (d + 31) / 32, parts = dt == SIGE_F32 ? Cache4Compute<float>::parts : 1;
    if (many && cache4_has_common(DT, parts)) return {32 * cache4_common_waves(DT), 1, 32 * cache4_common_tiles(DT)};
    return {32, many ? CACHE4_CROWD_WAVES : cache4_apart_waves(DT, parts), 32 * cache4_apart_tiles(DT, parts)};
}

// Waves of a workgroup.  Of more workgroups than compute units those with all waves fill the chip in few uneven rounds, and with few
// chunks leave most waves idle: as many waves as the chip holds at once by registers (heads from 136 on, single precision from 72 on: one
// per SIMD runs best), a power of two, none without a chunk (4096 queries of 77 tokens x 8 of 80 22 -> 9 us, of 160 25 -> 15; of 1500
// tokens x 80 43 -> 32, x 160 85 -> 72; the wrong way 1500 queries of 1500 x 160 42 -> 49); half types' heads from 136 on, to the nearest
// (1100 queries of 4000 x 8 of 160 110 us with two waves, 90 with four).  Where rows have ranges workgroups differ in length,
// and large ones end sooner (2889 rows with ranges of 12052 x 10 of 32 68 us, 88 with four waves).  Fewer workgroups than
// compute units: idle waves cost nothing, and all of them write.
static int cache4_waves(const Cache4Cut& cut, long workgroups, int share, bool many, bool ranges, bool wide)
{
    if (cut.waves == 1 || workgroups <= 256) return cut.waves;
    const double hold = ranges ? cut.waves : 256.0 * cut.waves * (many ? 4 : 1) / workgroups;
    int w = cut.waves;
    while (w > 1 && (w > (wide ? hold + hold / 3 : hold) || w / 2 >= share)) w /= 2;
    return w;
}

// room: floats of workspace, what the splits' partial sums have to fit into.
//
// Half types, from where on a call counts as one of many queries (heads x tiles of 32, "tiles"):
//   heads up to 64    more tiles than compute units: workgroups side by side (512 tiles of 1024 tokens x 40 13.5 against 15.9 us; 256 of
//                     3000 x 64 17.4 against 16.7)
//   larger heads      a product of tiles, tokens and d^2 beyond which common chunks win, within 10 % (d = 96: tiles x tokens 2^21 53
//                     against 42 us, 2^22 74.5 against 73.5; 128: 2^20 45 against 32, 2^21 55 against 56, 2^22 85 against 98; 160: 2^20 52
//                     against 50, 2^21 74 against 87; 256: 2^18 46 against 45, 2^19 55 against 47, 2^20 67 against 83); with ranges, of which 256
//                     rows span more than 32, up to d = 128 four times of it (1024 rows of 16384 x 8 of 96 76 against 85 us, of 128 69 against 94;
//                     2048 of 4096 x 8 of 128 63 against 59)
// Splits over workgroups: of one to six rounds of the chip (of common chunks up to d = 96 a compute unit holds three workgroups, else
// one) the number that costs least at 2.5 us per round, 2 per chunk (measured: 1.3 - 2.2 over all forms), and 3 and the partial sums'
// bytes for the merge (1500 queries of 16384 x 3 of 40, 141 tiles: 51 -> 39 us); none for fewer than four chunks per wave, which end
// before that (16 queries of 4096 x 8 of 40, eight chunks per wave: 16.2 us alone, 12.9, 10.0 and 9.0 in 2, 4 and 8 splits; 160 tiles of
// 4096 x 80 22.6 alone, 29.6 in two), nor side by
// side, nor where every wave has tiles enough by itself (more tiles than compute units).  Rows with ranges of their own make workgroups of different lengths: up to four
// (side by side: eight) times as many then, of eight chunks per wave at least (2379 rows with ranges of 20391 x 2 of 32 52 -> 31 us; 640
// of 4096 x 8 of 64 18.3, 22.5 in two of four chunks).
static Cache4Form plan_cache4(int Nq, int T, int heads, int d, sige_dtype dt, bool ranges, size_t room = ~(size_t)0)
{
    const int target = knob(SIGE_KNOB_ATTN_WGS);
    const long tiles = (long)heads * (((long)Nq + 31) / 32);
    const int many = knob(SIGE_KNOB_CACHE4_MANY);
    const bool crosses = d <= 64 ? tiles > 256 : (double)tiles * T * d * d >= (double)(1L << (ranges && d <= 128 ? 37 : 35));
    Cache4Form f = {dt != SIGE_F32 && (many >= 0 ? many != 0 : crosses), 1};
    const Cache4Cut cut = cache4_cut(d, dt, f.many);
    const long chunks = ((long)T + cut.chunk - 1) / cut.chunk;
    const long base = (long)heads * (((long)Nq + cut.rows - 1) / cut.rows);
    const long fill = cut.waves == 1 && d <= 96 ? 768 : 256;
    const bool crowd = f.many && cut.waves > 1;
    const long most = std::max(std::min(chunks / cut.waves, 64L), 1L);
    long want = target >= 0 ? (target + base - 1) / base : 1;
    if (target < 0 && !crowd && (cut.waves == 1 || base <= fill) && chunks >= 4 * cut.waves) {
        double least = INFINITY;
        for (int rounds = 1; rounds <= 6; ++rounds) {
            const long z = std::max(std::min(fill * rounds / base, most), 1L);
            const double cost = ((base * z + fill - 1) / fill) * (2.5 + 2.0 * ((chunks + z * cut.waves - 1) / (z * cut.waves))) +
                                (z > 1 ? 3.0 + 1.6e-6 * z * heads * Nq * (d + 4) : 0.0);
            if (cost < least) { least = cost; want = z; }
        }
    }
    if (target < 0 && ranges && cut.waves > 1) want = std::max(want, std::min((crowd ? 8 : 4) * fill / base, chunks / (8 * cut.waves)));
    want = std::max(std::min(want, most), 1L);
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
    SIGE_REQUIRE(T <= 0x7fffffff - 128, SIGE_ERR_UNSUPPORTED, "%s: too many tokens", who);       // (a chunk's end is an int)
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
    a.inv_scale = 1.0f / a.scale_log2e;
    a.d_heads = fast_div(heads); a.d_tpb = fast_div(a.q_tpb); a.d_qbw = fast_div(a.q_bw); a.d_dq = fast_div(d / 4);
    const bool room = workspace != nullptr && aligned16(workspace);
    const Cache4Form f = plan_cache4(Nq, T, heads, d, dt, ranges != nullptr, room ? workspace_bytes / sizeof(float) : 0);
    const Cache4Cut cut = cache4_cut(d, dt, f.many);
    a.splits = f.splits;
    a.share = (int)((((long)T + cut.chunk - 1) / cut.chunk + f.splits - 1) / f.splits);
    a.d_splits = fast_div(f.splits);
    a.waves = cache4_waves(cut, (((long)Nq + cut.rows - 1) / cut.rows) * heads * f.splits, a.share, f.many, ranges != nullptr,
                           dt != SIGE_F32 && d > 128);
    hipStream_t st = (hipStream_t)stream;
    return dt == SIGE_F32 ? launch_cache4_f32(a, f, st) : dt == SIGE_F16 ? launch_cache4_f16(a, f, st) : launch_cache4_bf16(a, f, st);
}

}  // namespace sige

using namespace sige;

extern "C" size_t sige_cache4_attn_workspace_bytes(int32_t Nq, int32_t T, int32_t heads, int32_t d)
{
    if (Nq <= 0 || T <= 0 || heads <= 0 || d <= 0 || d > 256) return 0;
    int splits = 1;
    for (sige_dtype dt : {SIGE_F16, SIGE_F32})
        for (bool ranges : {false, true}) splits = std::max(splits, plan_cache4(Nq, T, heads, d, dt, ranges).splits);
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
