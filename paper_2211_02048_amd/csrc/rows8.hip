// Rows of tokens held in 8 bits, beside the token-wise layers of an attention block on the gathered tokens (Sec. 3.2 "Extension to
// attention layers", Fig. "sige-attention"): storing, reading back, and the root-mean-square norm of models that have it, with the
// residual's addition before it and an output in 8 bits behind it.
#include "rows8.h"

namespace sige {

struct Rows8Args {
    const void* x;
    const void* residual;
    const float* gamma;
    void* total;
    void* y;
    unsigned char* q;
    unsigned char* s;
    Rows8 rows;
    int C, x_ld, res_ld, total_ld, y_ld, q_ld, s_ld;
    float eps;
    FastDiv d_chunks;
};

// The lane's vectors of a chunk (zeros behind C).
template <typename T>
__device__ __forceinline__ void load_chunk(const T* x, int lane, int left, uint4 (&raw)[ChunkShape<T>::V])
{
    constexpr int V = ChunkShape<T>::V, N = ChunkShape<T>::N;
#pragma unroll
    for (int h = 0; h < V; ++h) {
        const int c = V == 1 ? 8 * lane : 256 * h + N * lane;
        raw[h] = c < left ? *(const uint4*)(x + c) : make_uint4(0, 0, 0, 0);
    }
}

// Rows to 8 bits.  Bound by memory: s + 1 bytes per value (16384 rows of 5120 in fp16 47 us, 5.4 TB/s, in single precision 73 us, 5.75).  A wave takes 512 channels of a row, so
// that the maximum of a block stays within 16 lanes (four register exchanges) and the four scale bytes leave as one word.
template <typename T>
__global__ __launch_bounds__(256) void rows8_store_kernel(Rows8Args a)
{
    constexpr int V = ChunkShape<T>::V, N = ChunkShape<T>::N;
    const int lane = threadIdx.x & 63;
    int row, chunk;
    divmod(blockIdx.x * 4 + (threadIdx.x >> 6), a.d_chunks, row, chunk);
    if (row >= rows8_effective(a.rows)) return;
    const int left = a.C - chunk * ROW8_CHUNK;
    uint4 raw[V];
    load_chunk<T>((const T*)a.x + (long)row * a.x_ld + chunk * ROW8_CHUNK, lane, left, raw);
    float f[V][N];
#pragma unroll
    for (int h = 0; h < V; ++h) unpack<T>(raw[h], f[h]);
    store_chunk<T>(f, lane, left, a.q + (long)row * a.q_ld + chunk * ROW8_CHUNK, a.s + (long)row * a.s_ld + chunk * 4);
}

// Rows from 8 bits.  Bound by memory (the same rows 38 us, 6.6 TB/s, where what was just stored is partly in the last-level cache, 47 us where it
// is not; to single precision 76 us, 5.5 TB/s).
template <typename T>
__global__ __launch_bounds__(256) void rows8_load_kernel(Rows8Args a)
{
    constexpr int V = ChunkShape<T>::V, N = ChunkShape<T>::N;
    const int lane = threadIdx.x & 63;
    int row, chunk;
    divmod(blockIdx.x * 4 + (threadIdx.x >> 6), a.d_chunks, row, chunk);
    if (row >= rows8_effective(a.rows)) return;
    const int left = a.C - chunk * ROW8_CHUNK;
    const unsigned char* q = a.q + (long)row * a.q_ld + chunk * ROW8_CHUNK;
    const unsigned word = *(const unsigned*)(a.s + (long)row * a.s_ld + chunk * 4);
    T* y = (T*)a.y + (long)row * a.y_ld + chunk * ROW8_CHUNK;
#pragma unroll
    for (int h = 0; h < V; ++h) {
        const int c = V == 1 ? 8 * lane : 256 * h + 4 * lane;
        if (c >= left) continue;
        const float scale = scale_value(word >> (c / ROW8_BLOCK * 8) & 255u);
        unsigned w[N / 4];
        if constexpr (V == 1) {
            const uint2 u = *(const uint2*)(q + c);
            w[0] = u.x; w[1] = u.y;
        } else {
            w[0] = *(const unsigned*)(q + c);
        }
        float f[N];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
            f[4 * i] = lo[0] * scale; f[4 * i + 1] = lo[1] * scale; f[4 * i + 2] = hi[0] * scale; f[4 * i + 3] = hi[1] * scale;
        }
        *(uint4*)(y + c) = pack<T>(f);
    }
}

// h = round(x + residual), n = gamma * h / sqrt(mean(h^2) + eps), to the outputs that are asked for.  Bound by memory (16384 rows of 2560 in bf16 with a
// residual, its sum and the 8-bit output 55 to 58 us, 5.1 to 5.3 TB/s); a row stays in registers between the sum of squares (fp32) and the outputs.  W waves
// share a row, chunk w + W u of 512 channels each.
template <typename T, int NC, int W>
__global__ __launch_bounds__(256) void rows8_rms_kernel(Rows8Args a)
{
    constexpr int V = ChunkShape<T>::V, N = ChunkShape<T>::N;
    __shared__ float part[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = blockIdx.x * (4 / W) + wave / W, w = wave % W;
    const bool on = row < rows8_effective(a.rows);
    if (W == 1 && !on) return;
    const int chunks = (a.C + ROW8_CHUNK - 1) / ROW8_CHUNK;
    float f[NC][V][N];
    float sum = 0.0f;
    uint4 raw[NC][V], add[NC][V];
    // every load of the row on its way before the first is waited for
#pragma unroll
    for (int u = 0; u < NC; ++u) {
        const int chunk = w + W * u, left = on && chunk < chunks ? a.C - chunk * ROW8_CHUNK : 0;
        load_chunk<T>((const T*)a.x + (long)row * a.x_ld + chunk * ROW8_CHUNK, lane, left, raw[u]);
    }
    if (a.residual) {
#pragma unroll
        for (int u = 0; u < NC; ++u) {
            const int chunk = w + W * u, left = on && chunk < chunks ? a.C - chunk * ROW8_CHUNK : 0;
            load_chunk<T>((const T*)a.residual + (long)row * a.res_ld + chunk * ROW8_CHUNK, lane, left, add[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < NC; ++u) {
        const int chunk = w + W * u, left = on && chunk < chunks ? a.C - chunk * ROW8_CHUNK : 0;
#pragma unroll
        for (int h = 0; h < V; ++h) {
            unpack<T>(raw[u][h], f[u][h]);
            if (a.residual) {
                float g[N];
                unpack<T>(add[u][h], g);
#pragma unroll
                for (int i = 0; i < N; ++i) f[u][h][i] += g[i];
                const uint4 t = pack<T>(f[u][h]);                // the sum is a stored tensor of the model's type, and the norm is that tensor's
                unpack<T>(t, f[u][h]);
                const int c = V == 1 ? 8 * lane : 256 * h + N * lane;
                if (a.total && c < left) *(uint4*)((T*)a.total + (long)row * a.total_ld + chunk * ROW8_CHUNK + c) = t;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sum = fmaf(f[u][h][i], f[u][h][i], sum);
        }
    }
    const auto over_row = [&] {
#pragma unroll
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        if constexpr (W > 1) {
            if (lane == 0) part[wave] = sum;
            __syncthreads();
            sum = part[0];
#pragma unroll
            for (int i = 1; i < W; ++i) sum += part[i];
        }
    };
    over_row();
    if (W > 1 && !on) return;                                // (four waves: the workgroup's one row)
    // Squares below fp32's normal numbers lose bits, or all of them, where eps does not hide them; above them the sum is infinite.  Such a row
    // is taken times a power of two, and eps with it: the quotient is the same, and what falls below the range now is 2^-100 of the largest.
    float eps = a.eps;
    const float by = sum < 0x1p-110f && eps < 0x1p-80f ? 0x1p100f : sum == __uint_as_float(0x7f800000u) ? 0x1p-80f : 1.0f;
    if (by != 1.0f) {
        eps = eps * by * by;
        sum = 0.0f;
#pragma unroll
        for (int u = 0; u < NC; ++u)
#pragma unroll
            for (int h = 0; h < V; ++h)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    f[u][h][i] *= by;
                    sum = fmaf(f[u][h][i], f[u][h][i], sum);
                }
        if constexpr (W > 1) __syncthreads();                // (every wave has read the parts)
        over_row();
    }
    const float r = 1.0f / sqrtf(sum / (float)a.C + eps);
#pragma unroll
    for (int u = 0; u < NC; ++u) {
        const int chunk = w + W * u;
        if (chunk >= chunks) continue;
        const int left = a.C - chunk * ROW8_CHUNK;
#pragma unroll
        for (int h = 0; h < V; ++h) {
            const int c = V == 1 ? 8 * lane : 256 * h + N * lane;
            if (c < left) {
                float g[N];
                if (a.gamma) load_f32_run<N>(a.gamma, chunk * ROW8_CHUNK + c, g);
#pragma unroll
                for (int i = 0; i < N; ++i) f[u][h][i] = a.gamma ? f[u][h][i] * r * g[i] : f[u][h][i] * r;
                if (a.y) *(uint4*)((T*)a.y + (long)row * a.y_ld + chunk * ROW8_CHUNK + c) = pack<T>(f[u][h]);
            }
        }
        if (a.q) store_chunk<T>(f[u], lane, left, a.q + (long)row * a.q_ld + chunk * ROW8_CHUNK, a.s + (long)row * a.s_ld + chunk * 4);
    }
}

// Checks of a tensor of rows of C values of dt.
static int check_tensor(const char* who, const char* what, const void* x, sige_dtype dt, int C, int ld, bool used)
{
    const int vw = (int)(16 / dtype_size(dt));
    SIGE_REQUIRE(ld >= C, SIGE_ERR_INVALID_ARG, "%s: the row stride of %s is below the %d channels", who, what, C);
    SIGE_REQUIRE(C % vw == 0 && ld % vw == 0, SIGE_ERR_UNSUPPORTED, "%s: the channels and the row stride of %s must be multiples of %d", who, what, vw);
    if (!used) return SIGE_OK;
    SIGE_REQUIRE(x, SIGE_ERR_INVALID_ARG, "%s: %s is required", who, what);
    SIGE_REQUIRE(aligned16(x), SIGE_ERR_UNSUPPORTED, "%s: %s must be 16-byte aligned", who, what);
    return SIGE_OK;
}

}  // namespace sige

using namespace sige;

static int rows8_store_load(const char* who, bool store, void* x, sige_dtype dt, int32_t C, int32_t x_ld, const int32_t* count,
                            int32_t rows_per_count, int32_t max_rows, int32_t n_rows, void* q, int32_t q_ld, void* s, int32_t s_ld, void* stream)
{
    clear_error();
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    SIGE_REQUIRE(C > 0, SIGE_ERR_INVALID_ARG, "%s: need C > 0", who);
    Rows8Args a = {};
    int rows;
    if (int rc = rows8_check(who, count, rows_per_count, max_rows, n_rows, &a.rows, &rows)) return rc;
    if (int rc = check_tensor(who, store ? "x" : "y", x, dt, C, x_ld, rows > 0)) return rc;
    if (int rc = rows8_check_matrix(who, "the 8-bit rows", q, q_ld, s, s_ld, C, rows > 0)) return rc;
    if (rows == 0) return SIGE_OK;
    a.x = x; a.y = x; a.x_ld = a.y_ld = x_ld; a.C = C; a.q = (unsigned char*)q; a.q_ld = q_ld; a.s = (unsigned char*)s; a.s_ld = s_ld;
    const int chunks = (int)(((long)C + ROW8_CHUNK - 1) / ROW8_CHUNK);       // (C + 511 need not fit an int)
    a.d_chunks = fast_div(chunks);
    const long waves = (long)rows * chunks;
    SIGE_REQUIRE(waves <= ROW8_MOST_WAVES, SIGE_ERR_UNSUPPORTED, "%s: at most 2^26 - 4 rows, counted once for every 512 channels begun", who);
    // (a wave writes a chunk while others still read the rows around it)
    SIGE_REQUIRE(q != x && s != x && q != s, SIGE_ERR_INVALID_ARG, "%s: the 8-bit rows in the place of %s or of each other", who, store ? "x" : "y");
    const dim3 grid((unsigned)((waves + 3) / 4));
    hipStream_t st = (hipStream_t)stream;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, grid, dim3(256), 0, st, a); };
    if (store) {
        if (dt == SIGE_F32) go(rows8_store_kernel<float>);
        else if (dt == SIGE_F16) go(rows8_store_kernel<f16>);
        else go(rows8_store_kernel<bf16>);
    } else {
        if (dt == SIGE_F32) go(rows8_load_kernel<float>);
        else if (dt == SIGE_F16) go(rows8_load_kernel<f16>);
        else go(rows8_load_kernel<bf16>);
    }
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

extern "C" int sige_rows8_store(const void* x, sige_dtype dt, int32_t C, int32_t x_ld, const int32_t* count, int32_t rows_per_count,
                                int32_t max_rows, int32_t n_rows, void* q, int32_t q_ld, void* scales, int32_t s_ld, void* stream)
{
    return rows8_store_load("sige_rows8_store", true, const_cast<void*>(x), dt, C, x_ld, count, rows_per_count, max_rows, n_rows, q, q_ld, scales, s_ld, stream);
}

extern "C" int sige_rows8_load(const void* q, int32_t q_ld, const void* scales, int32_t s_ld, int32_t C, const int32_t* count,
                               int32_t rows_per_count, int32_t max_rows, int32_t n_rows, void* y, sige_dtype dt, int32_t y_ld, void* stream)
{
    return rows8_store_load("sige_rows8_load", false, y, dt, C, y_ld, count, rows_per_count, max_rows, n_rows, const_cast<void*>(q), q_ld,
                            const_cast<void*>(scales), s_ld, stream);
}

extern "C" int sige_token_rms(const void* x, sige_dtype dt, int32_t C, int32_t x_ld, const void* residual, int32_t res_ld, const int32_t* count,
                              int32_t rows_per_count, int32_t max_rows, int32_t n_rows, const float* gamma, float eps, void* total,
                              int32_t total_ld, void* y, int32_t y_ld, void* q, int32_t q_ld, void* scales, int32_t s_ld, void* stream)
{
    clear_error();
    const char* who = "sige_token_rms";
    SIGE_REQUIRE(dtype_ok(dt), SIGE_ERR_INVALID_ARG, "%s: unknown dtype %d", who, (int)dt);
    SIGE_REQUIRE(C > 0 && eps >= 0.0f, SIGE_ERR_INVALID_ARG, "%s: need C > 0 and eps >= 0", who);
    Rows8Args a = {};
    int rows;
    if (int rc = rows8_check(who, count, rows_per_count, max_rows, n_rows, &a.rows, &rows)) return rc;
    // (without rows a tensor's address may be null: which tensors there are says nothing)
    SIGE_REQUIRE(y || q || rows == 0, SIGE_ERR_INVALID_ARG, "%s: y or the 8-bit rows are required", who);
    SIGE_REQUIRE(residual || !total || rows == 0, SIGE_ERR_INVALID_ARG, "%s: the sum is an output beside a residual only", who);
    if (int rc = check_tensor(who, "x", x, dt, C, x_ld, rows > 0)) return rc;
    if (residual)
        if (int rc = check_tensor(who, "residual", residual, dt, C, res_ld, rows > 0)) return rc;
    if (total)
        if (int rc = check_tensor(who, "total", total, dt, C, total_ld, rows > 0)) return rc;
    if (y)
        if (int rc = check_tensor(who, "y", y, dt, C, y_ld, rows > 0)) return rc;
    if (q)
        if (int rc = rows8_check_matrix(who, "the 8-bit rows", q, q_ld, scales, s_ld, C, rows > 0)) return rc;
    SIGE_REQUIRE(C * dtype_size(dt) <= 32768, SIGE_ERR_UNSUPPORTED, "%s: at most 32 KiB per token", who);
    SIGE_REQUIRE((reinterpret_cast<uintptr_t>(gamma) & 3u) == 0, SIGE_ERR_UNSUPPORTED, "%s: gamma must be 4-byte aligned", who);
    if (rows == 0) return SIGE_OK;
    // (a wave writes a row's sums where it has read that row, and only that row's)
    SIGE_REQUIRE((total != x || total_ld == x_ld) && (total != residual || !total || total_ld == res_ld) && (y != x || y_ld == x_ld) &&
                     (!residual || y != residual || y_ld == res_ld),
                 SIGE_ERR_UNSUPPORTED, "%s: an output in the place of an input needs its row stride", who);
    SIGE_REQUIRE(!total || total != y, SIGE_ERR_INVALID_ARG, "%s: the sum and y are two outputs", who);
    SIGE_REQUIRE(!gamma || (total != gamma && y != gamma && q != gamma && scales != gamma), SIGE_ERR_INVALID_ARG,
                 "%s: an output in the place of gamma", who);
    a.x = x; a.residual = residual; a.gamma = gamma; a.total = total; a.y = y; a.q = (unsigned char*)q; a.s = (unsigned char*)scales;
    a.C = C; a.x_ld = x_ld; a.res_ld = res_ld; a.total_ld = total_ld; a.y_ld = y_ld; a.q_ld = q_ld; a.s_ld = s_ld; a.eps = eps;
    const int chunks = (C + ROW8_CHUNK - 1) / ROW8_CHUNK;
    SIGE_REQUIRE((long)rows * chunks <= ROW8_MOST_WAVES, SIGE_ERR_UNSUPPORTED, "%s: at most 2^26 - 4 rows, counted once for every 512 channels begun", who);
    for (const void* p : {(const void*)q, (const void*)scales})
        SIGE_REQUIRE(!q || (p != x && p != residual && p != total && p != y && q != scales), SIGE_ERR_INVALID_ARG,
                     "%s: the 8-bit rows in the place of another tensor or of each other", who);
    // (single precision, three chunks: a workgroup of 256 threads per row; every other form has fewer than 2^32 threads by the limit above)
    SIGE_REQUIRE(dt != SIGE_F32 || chunks <= 2 || rows < (1 << 24), SIGE_ERR_UNSUPPORTED, "%s: fewer than 2^24 rows of more than 1024 channels in single precision", who);
    hipStream_t st = (hipStream_t)stream;
    auto go = [&](auto kern, int W) { hipLaunchKernelGGL(kern, dim3((unsigned)(((long)rows * W + 3) / 4)), dim3(256), 0, st, a); };
    auto pick = [&](auto t) {
        using T = decltype(t);
        constexpr bool F = sizeof(T) == 4;
        constexpr int MOST = F ? 2 : 4;                        // chunks that one wave takes
        // a row of up to 2048 channels: four waves where rows are few (bf16, 256 rows of 1280 4.5 -> 3.0 us, of 2048 5.1 -> 3.0), one where they
        // are many (16384 of 1280 23.8 -> 22.9) unless its values are wide (single precision, 16384 of 2048 59 -> 56 by four)
        if (chunks <= 1) go(rows8_rms_kernel<T, 1, 1>, 1);
        else if (chunks <= 4 && (rows <= 2048 || (F && chunks > 2))) go(rows8_rms_kernel<T, 1, 4>, 4);
        else if (chunks <= 2) go(rows8_rms_kernel<T, 2, 1>, 1);
        else if (chunks <= MOST) go(rows8_rms_kernel<T, MOST, 1>, 1);
        else if (chunks <= 8) go(rows8_rms_kernel<T, 2, 4>, 4);
        else if (chunks <= 16) go(rows8_rms_kernel<T, 4, 4>, 4);
        else if constexpr (!F) go(rows8_rms_kernel<T, 8, 4>, 4);
    };
    if (dt == SIGE_F32) pick(float());
    else if (dt == SIGE_F16) pick(f16());
    else pick(bf16());
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}
