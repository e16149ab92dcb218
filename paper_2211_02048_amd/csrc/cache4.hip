// sige_cache4_store / sige_cache4_load: rows of keys and values into the cache held in 4 bits, and back.
// (The paper keeps the keys and values of the original image for every attention layer, Fig. "sige-attention": the cache is what
// a server of many images has in memory, a quarter of it in this form.)
//
// Both are bound by memory: a value is 2 or 4 bytes on one side and 0.53 on the other, and four instructions.  Four lanes share a
// group of 32 channels (16 bytes of a half-type row each) and 16 tokens lie side by side in a wave, so that it reads 64 whole
// bytes of 16 rows and writes 256 bytes of one plane in a run.  Measured: 16384 tokens of 8 heads of 128 in fp16, stored 23.6 us, read back
// 15.9 us, 85 MB each, 3.6 and 5.3 TB/s (a large copy reaches 5.2); 640 tokens of 8 heads of 40 2.4 us each, which is a launch.  (The single
// scale bytes make 51 MB of the 18 that a store writes; a wave with all groups of a head, which writes them in one piece, takes as long, and
// 15 - 30 % longer on few rows.)
#include "cache4.h"

namespace sige {

struct Cache4Rows {
    const void* k;
    const void* v;
    void* ko;
    void* vo;
    uint8_t* cache;
    const int32_t* slots;
    const int32_t* indices;    // rows are the pixels of listed blocks (token first + y * W + x)
    const int32_t* count;
    Cache4Layout l;
    int k_ld, v_ld, heads, d, groups, capacity, first;
    int rows_per_count, max_rows, n_host;
    int bw, H, W;
    FastDiv d_pb, d_bw, d_units, d_groups;
};

// Where row r goes: its token, or -1.
__device__ __forceinline__ int cache4_token(const Cache4Rows& a, int row)
{
    long t;
    if (a.indices != nullptr) {
        int b, p, py, px;
        divmod(row, a.d_pb, b, p);
        divmod(p, a.d_bw, py, px);
        const int y = a.indices[2 * b] + py, x = a.indices[2 * b + 1] + px;
        if (y < 0 || y >= a.H || x < 0 || x >= a.W) return -1;
        t = a.first + (long)y * a.W + x;
    } else {
        t = a.slots != nullptr ? (long)a.slots[row] : (long)a.first + row;
    }
    return t >= 0 && t < a.capacity ? (int)t : -1;
}

template <typename T>
__global__ __launch_bounds__(256) void cache4_store_kernel(Cache4Rows a)
{
    constexpr bool HALF = __is_same(T, f16);
    const int lane = threadIdx.x & 63, part = lane & 3, sub = lane >> 2;
    // a wave's 16 rows and its group: of a row tile all groups of all heads, keys and values, follow each other
    const unsigned wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    int tile, unit, hw, g;
    divmod((int)wave, a.d_units, tile, unit);
    divmod(unit, a.d_groups, hw, g);
    const int which = hw >= a.heads, head = hw - (which ? a.heads : 0);
    long rows = a.n_host;
    if (a.n_host < 0) {
        rows = (long)(*a.count) * a.rows_per_count;
        if (rows > a.max_rows) rows = a.max_rows;
    }
    const long row = (long)tile * 16 + sub;
    const bool live = row < rows;
    const int token = live ? cache4_token(a, (int)row) : -1;
    const int ch = 32 * g + 8 * part;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.0f;
    if (token >= 0 && ch < a.d) {
        const T* src = (const T*)(which ? a.v : a.k) + row * (which ? a.v_ld : a.k_ld) + head * a.d + ch;
        if constexpr (sizeof(T) == 4) {
            unpack<float>(*(const uint4*)src, f);
            unpack<float>(*(const uint4*)(src + 4), f + 4);
        } else {
            unpack<T>(*(const uint4*)src, f);
        }
    }
    // the largest magnitude by its bits: infinities and NaN are above every number
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
    top = max(top, (unsigned)__shfl_xor((int)top, 1));
    top = max(top, (unsigned)__shfl_xor((int)top, 2));
    if (token < 0) return;
    // the smallest power of two with top <= 6 * 2^e (top = m 2^x: e = x - 2, or x - 1 where m > 1.5): nothing is clipped, but where
    // e is held within what the rows' type can hold
    const bool finite = top < 0x7f800000u;
    int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
    e = min(max(e, HALF ? CACHE4_F16_E_MIN : CACHE4_E_MIN), HALF ? CACHE4_F16_E_MAX : CACHE4_E_MAX);
    unsigned w = 0;
    if (finite) {
        const float scale = cache4_scale((unsigned)(e + 127));
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[0], f[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[2], f[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[4], f[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f[6], f[7], scale, 3);
    }
    uint8_t* sec = a.cache + (2L * head + which) * a.l.section;
    if (g < a.l.full) *(unsigned*)(sec + (g * a.l.cap + token) * 16 + 4 * part) = w;
    else if (part < 2) *(unsigned*)(sec + a.l.full * a.l.cap * 16 + token * 8L + 4 * part) = w;
    if (part == 0) sec[a.l.scales + ((long)token << a.l.gs_log2) + g] = (uint8_t)(finite ? e + 127 : 255);
}

template <typename T>
__global__ __launch_bounds__(256) void cache4_load_kernel(Cache4Rows a)
{
    const int lane = threadIdx.x & 63, part = lane & 3, sub = lane >> 2;
    const unsigned wave = blockIdx.x * 4 + (threadIdx.x >> 6);
    int tile, unit, hw, g;
    divmod((int)wave, a.d_units, tile, unit);
    divmod(unit, a.d_groups, hw, g);
    const int which = hw >= a.heads, head = hw - (which ? a.heads : 0);
    const long row = (long)tile * 16 + sub;
    const int ch = 32 * g + 8 * part;
    T* out = (T*)(which ? a.vo : a.ko);
    if (row >= a.n_host || ch >= a.d || out == nullptr) return;
    const long token = a.first + row;
    const uint8_t* sec = a.cache + (2L * head + which) * a.l.section;
    const unsigned w = g < a.l.full ? *(const unsigned*)(sec + (g * a.l.cap + token) * 16 + 4 * part)
                                    : *(const unsigned*)(sec + a.l.full * a.l.cap * 16 + token * 8 + 4 * part);
    const unsigned byte = sec[a.l.scales + (token << a.l.gs_log2) + g];
    const float scale = byte > (__is_same(T, f16) ? CACHE4_F16_LAST : CACHE4_LAST) ? NAN : cache4_scale(byte);
    float f[8];
#define SIGE_CACHE4_TWO(s)                                                                     \
    {                                                                                          \
        const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, s);                   \
        f[2 * s] = p[0] * scale;                                                               \
        f[2 * s + 1] = p[1] * scale;                                                           \
    }
    SIGE_CACHE4_TWO(0) SIGE_CACHE4_TWO(1) SIGE_CACHE4_TWO(2) SIGE_CACHE4_TWO(3)
#undef SIGE_CACHE4_TWO
    T* dst = out + row * (which ? a.v_ld : a.k_ld) + head * a.d + ch;
    if constexpr (sizeof(T) == 4) {
        *(uint4*)dst = pack<float>(f);
        *(uint4*)(dst + 4) = pack<float>(f + 4);
    } else {
        *(uint4*)dst = pack<T>(f);
    }
}

static int check_cache4(const char* who, sige_dtype dt, int heads, int d, const void* cache, int capacity)
{
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    SIGE_REQUIRE(heads > 0 && d > 0 && capacity > 0, SIGE_ERR_INVALID_ARG, "%s: need heads > 0, d > 0, capacity > 0", who);
    SIGE_REQUIRE(d % 8 == 0 && d <= 256, SIGE_ERR_UNSUPPORTED, "%s: d must be a multiple of 8 and <= 256", who);
    SIGE_REQUIRE(heads <= 65535, SIGE_ERR_UNSUPPORTED, "%s: too many heads", who);
    SIGE_REQUIRE(cache != nullptr, SIGE_ERR_INVALID_ARG, "%s: the cache is required", who);
    SIGE_REQUIRE(aligned16(cache), SIGE_ERR_UNSUPPORTED, "%s: the cache must be 16-byte aligned", who);
    return SIGE_OK;
}

static int check_row(const char* who, const void* p, int ld, sige_dtype dt, int heads, int d, const char* name)
{
    const int vw = dt == SIGE_F32 ? 4 : 8;
    SIGE_REQUIRE(ld >= (long)heads * d, SIGE_ERR_INVALID_ARG, "%s: the row stride of %s must be >= heads*d", who, name);
    SIGE_REQUIRE(ld % vw == 0 && aligned16(p), SIGE_ERR_UNSUPPORTED,
                 "%s: the row stride of %s must be a multiple of %d elements, its pointer 16-byte aligned", who, name, vw);
    return SIGE_OK;
}

static void fill_rows(Cache4Rows& a, const void* cache, int capacity, int heads, int d)
{
    a.cache = (uint8_t*)cache;
    a.capacity = capacity; a.heads = heads; a.d = d;
    a.l = cache4_layout(d, capacity);
    a.groups = a.l.full + a.l.tail;
    a.d_units = fast_div(2 * heads * a.groups);
    a.d_groups = fast_div(a.groups);
    a.slots = a.indices = a.count = nullptr;
    a.k = a.v = nullptr; a.ko = a.vo = nullptr;
    a.rows_per_count = a.max_rows = 0;
    a.bw = a.H = a.W = 1;
    a.d_pb = a.d_bw = fast_div(1);
}

static int launch_rows(const char* who, const Cache4Rows& a, sige_dtype dt, int rows, bool store, hipStream_t st)
{
    const long waves = ((long)rows + 15) / 16 * (2L * a.heads * a.groups);
    SIGE_REQUIRE(waves < (1L << 26) - 4, SIGE_ERR_UNSUPPORTED, "%s: too many rows", who);     // (a launch has 2^32 threads)
    const dim3 grid((unsigned)((waves + 3) / 4));
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
    if (store) {
        if (dt == SIGE_F32) go(cache4_store_kernel<float>);
        else if (dt == SIGE_F16) go(cache4_store_kernel<f16>);
        else go(cache4_store_kernel<bf16>);
    } else {
        if (dt == SIGE_F32) go(cache4_load_kernel<float>);
        else if (dt == SIGE_F16) go(cache4_load_kernel<f16>);
        else go(cache4_load_kernel<bf16>);
    }
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

}  // namespace sige

using namespace sige;

extern "C" size_t sige_cache4_bytes(int32_t heads, int32_t d, int32_t capacity)
{
    if (heads <= 0 || heads > 65535 || d <= 0 || d % 8 != 0 || d > 256 || capacity <= 0) return 0;
    return (size_t)cache4_layout(d, capacity).section * 2 * heads;
}

extern "C" int sige_cache4_store(const void* k, int32_t k_ld, const void* v, int32_t v_ld, sige_dtype dt, int32_t heads,
                                 int32_t d, const int32_t* slots, int32_t first, const int32_t* count, int32_t rows_per_count,
                                 int32_t max_rows, int32_t n_rows, void* cache, int32_t capacity, void* stream)
{
    clear_error();
    const char* who = "sige_cache4_store";
    if (int rc = check_cache4(who, dt, heads, d, cache, capacity)) return rc;
    SIGE_REQUIRE(k && v, SIGE_ERR_INVALID_ARG, "%s: k and v are required", who);
    if (int rc = check_row(who, k, k_ld, dt, heads, d, "k")) return rc;
    if (int rc = check_row(who, v, v_ld, dt, heads, d, "v")) return rc;
    SIGE_REQUIRE(max_rows >= 0 && n_rows >= -1 && n_rows <= max_rows, n_rows > max_rows ? SIGE_ERR_CAPACITY : SIGE_ERR_INVALID_ARG,
                 "%s: need 0 <= n_rows <= max_rows (or n_rows = -1)", who);
    SIGE_REQUIRE(n_rows >= 0 || (count != nullptr && rows_per_count > 0), SIGE_ERR_INVALID_ARG,
                 "%s: count and rows_per_count are required when n_rows is -1", who);
    SIGE_REQUIRE(first >= 0 && (first == 0 || slots == nullptr), SIGE_ERR_INVALID_ARG, "%s: first is a token >= 0, and 0 beside slots", who);
    // (a device count may name fewer rows than the host allows: rows past the capacity are skipped there, refused here)
    SIGE_REQUIRE(slots != nullptr || n_rows < 0 || (long)first + n_rows <= capacity, SIGE_ERR_CAPACITY,
                 "%s: %d rows from token %d exceed the capacity (%d)", who, n_rows, first, capacity);
    const int rows = n_rows >= 0 ? n_rows : max_rows;
    if (rows == 0) return SIGE_OK;
    Cache4Rows a;
    fill_rows(a, cache, capacity, heads, d);
    a.k = k; a.v = v; a.k_ld = k_ld; a.v_ld = v_ld;
    a.slots = slots; a.first = first; a.count = count; a.rows_per_count = rows_per_count; a.max_rows = max_rows; a.n_host = n_rows;
    return launch_rows(who, a, dt, rows, true, (hipStream_t)stream);
}

extern "C" int sige_cache4_store_blocks(const void* k, int32_t k_ld, const void* v, int32_t v_ld, sige_dtype dt, int32_t heads,
                                        int32_t d, const sige_geom* g, const int32_t* indices, const int32_t* count,
                                        int32_t max_blocks, int32_t n_blocks, int32_t first, void* cache, int32_t capacity,
                                        void* stream)
{
    clear_error();
    const char* who = "sige_cache4_store_blocks";
    int nl;
    if (int rc = check_geom(g, who, nullptr, nullptr)) return rc;
    if (int rc = check_blocks(count, max_blocks, n_blocks, who, &nl)) return rc;
    if (int rc = check_cache4(who, dt, heads, d, cache, capacity)) return rc;
    SIGE_REQUIRE(g->k == 1 && g->stride == 1 && g->pad == 0, SIGE_ERR_UNSUPPORTED,
                 "%s: tokens are the pixels of the blocks themselves (k = 1, stride 1, no padding)", who);
    SIGE_REQUIRE(k && v && indices, SIGE_ERR_INVALID_ARG, "%s: k, v and indices are required", who);
    if (int rc = check_row(who, k, k_ld, dt, heads, d, "k")) return rc;
    if (int rc = check_row(who, v, v_ld, dt, heads, d, "v")) return rc;
    SIGE_REQUIRE(first >= 0 && first + (long)g->H_in * g->W_in <= capacity, SIGE_ERR_CAPACITY,
                 "%s: a map of %d x %d tokens from token %d exceeds the capacity (%d)", who, g->H_in, g->W_in, first, capacity);
    const long pb = (long)g->block_h * g->block_w;
    SIGE_REQUIRE(pb * max_blocks < (1L << 31), SIGE_ERR_UNSUPPORTED, "%s: too many tokens", who);
    if (nl == 0) return SIGE_OK;
    Cache4Rows a;
    fill_rows(a, cache, capacity, heads, d);
    a.k = k; a.v = v; a.k_ld = k_ld; a.v_ld = v_ld;
    a.indices = indices; a.first = first; a.count = count; a.rows_per_count = (int)pb; a.max_rows = (int)(pb * max_blocks);
    a.n_host = n_blocks >= 0 ? (int)(pb * n_blocks) : -1;
    a.bw = g->block_w; a.H = g->H_in; a.W = g->W_in;
    a.d_pb = fast_div((int)pb); a.d_bw = fast_div(g->block_w);
    return launch_rows(who, a, dt, (int)(pb * nl), true, (hipStream_t)stream);
}

extern "C" int sige_cache4_load(const void* cache, int32_t capacity, sige_dtype dt, int32_t heads, int32_t d, int32_t first,
                                int32_t n_tokens, void* k, int32_t k_ld, void* v, int32_t v_ld, void* stream)
{
    clear_error();
    const char* who = "sige_cache4_load";
    if (int rc = check_cache4(who, dt, heads, d, cache, capacity)) return rc;
    SIGE_REQUIRE(k || v, SIGE_ERR_INVALID_ARG, "%s: k or v is required", who);
    if (k) if (int rc = check_row(who, k, k_ld, dt, heads, d, "k")) return rc;
    if (v) if (int rc = check_row(who, v, v_ld, dt, heads, d, "v")) return rc;
    SIGE_REQUIRE(first >= 0 && n_tokens >= 0, SIGE_ERR_INVALID_ARG, "%s: first and n_tokens must not be negative", who);
    SIGE_REQUIRE((long)first + n_tokens <= capacity, SIGE_ERR_CAPACITY, "%s: tokens %d..%ld exceed the capacity (%d)", who, first,
                 (long)first + n_tokens - 1, capacity);
    if (n_tokens == 0) return SIGE_OK;
    Cache4Rows a;
    fill_rows(a, cache, capacity, heads, d);
    a.ko = k; a.vo = v; a.k_ld = k_ld; a.v_ld = v_ld; a.first = first; a.n_host = n_tokens;
    return launch_rows(who, a, dt, n_tokens, false, (hipStream_t)stream);
}
