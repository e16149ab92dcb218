// The product of two matrices in 8 bits for many rows: tiles of 64 RT rows x 64 CT output channels, four waves of 32 RT x 32 CT each.
//
// Bound by the matrix pipes for large calls.  v_mfma_scale_f32_32x32x64_f8f6f4 (weights as its first operand, so that a lane holds consecutive
// channels of one token; its two scales are those of the block of 128 channels that its 64 lie in).  A block of 128 channels of both operands
// comes into LDS by direct loads, whole 128-byte lines (halves of lines took 1.4 times as long: twice the requests), NS blocks
// deep; the 16-byte pieces of a row are permuted by the row's number, so that neither the loads nor the reads meet in a bank.  While the
// pipe works on one half of a block, the next half's operands are read into registers, one read or request between two
// matrix instructions: there is one wave per SIMD in the largest form, and whatever it waits for the pipe waits for too (in a
// prototype, 8192 x 8192 x 8192: requests in one burst 2565 TFLOP/s, spread 2750).  No branch in the loop: the compiler moves matrix instructions behind it (2040).
// Measured, inputs changing: 8192 x 8192 -> 8192 409 us, 2690 TFLOP/s (inputs in the cache 390; all codes 0 331 and 289: the clock is at 1.9 GHz
// of 2.4 for power); 8192 x 5120 -> 5120 184 us, 2340 TFLOP/s, with a base matrix pipes busy 58 % of all cycles, LDS 18 %.
// Single precision, whose codes are expanded to bf16 on their way into the pipes: 915 us, 1200 TFLOP/s, and 380 us, 1130.
#pragma once

#include "rows8_linear.h"

namespace sige {

constexpr int COMPUTE_UNITS = 256;

// LDS rows of the weights: which output channel of the wave's (of its values and of its gates, if gated) lies at place p of the tile.  In the
// result, place 8 (r / 4) + 4 h + r % 4 of 32 is in register r of the lanes of half h.
template <bool GATED>
__device__ __forceinline__ int tile_channel(int p)
{
    const int u = p & 31;
    if (!GATED)         // registers 8 v .. 8 v + 7: channels 16 v + 8 h ...
        return (p & ~31) + 16 * (u >> 4) + 8 * (u >> 2 & 1) + 4 * (u >> 3 & 1) + (u & 3);
    // (four tiles of 32 per wave: two of values, two of their gates; tile t's registers: channels 32 h + 16 t ...)
    return (p >> 7) * 64 + 32 * (u >> 2 & 1) + 16 * (p >> 5 & 1) + 4 * (u >> 3) + (u & 3);
}

template <typename T, bool GATED, int RT, int CT, int NS>
struct Tile8 {
    static constexpr bool EXACT = sizeof(T) == 4;
    static constexpr int BM = 64 * RT, BN = 64 * CT, OUT = GATED ? BN / 2 : BN;          // rows, weight rows and output channels of a tile
    static constexpr int XB = BM * 128, STAGE = XB + BN * 128, SC = NS * STAGE;          // bytes in LDS; where the scale words are
    static constexpr int XI = BM / 32, WI = BN / 32, REQ = XI + WI;                      // direct loads of a wave per block
    // (gated: requests i and i ^ 2 are for values and gates of the same channels; each kind's rows are counted from its own first one, so that
    // the offsets do not have to hold the way from one to the other)
    static constexpr int WO = GATED ? WI / 2 : WI;
    static constexpr int wo_of(int i) { return GATED ? (i & 1) | i >> 2 << 1 : i; }
    static constexpr int N = RT * CT;                                                    // matrix instructions of a wave per half block
    // a block's 2 N matrix instructions are its time: operands of its second half are read beside the first of them, READS at a time; behind
    // number FREE its place is requested into again, PER requests at a time, and at number COME the next block has to have come
    static constexpr int READS = (RT + CT + N - 1) / N, READ = (RT + CT + READS - 1) / READS;
    static constexpr int FREE = READ + (N >= 16 ? 2 : N >= 8 ? 1 : 0), COME = 2 * N - READ - (N >= 16 ? 2 : 0);
    static constexpr int PER = (REQ + 2 * N - FREE - 1) / (2 * N - FREE);
    static_assert(FREE <= COME && COME >= N, "");
    static constexpr int GROUPS = (BM + BN) / 64;                                        // of scale words, 64 rows each
    static constexpr int EPI = SC + 4 * (BM + BN) * 4, LDS = EPI + BN * 4 + (GATED ? 2 * BM * 4 : 0);   // four scale words of every row; bias, rows' maxima

    static __device__ __forceinline__ void mma(const i32x8& w, unsigned ws, const i32x8& x, unsigned xs, f32x16& c)
    {
        if constexpr (!EXACT) {
            c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, x, c, 0, 0, 0, (int)ws, 0, (int)xs);
        } else {
            const float fw = scale_value(ws & 255u), fx = scale_value(xs & 255u);
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(expand8(w[i], w[i + 1], fw), expand8(x[i], x[i + 1], fx), c, 0, 0, 0);
        }
    }

    // Where a tile's operands come from.
    struct Source {
        int row0, col0, rows, cols;                          // of the tile (rows and output channels that are there)
        int xo[XI], wo[WO];                                  // a lane's places in the tile's rows, for each of its requests per block
        const unsigned char* sp[2];                          // its scale words
        float bias;                                          // thread t's: that of the t-th row of weights of the tile, in the order of the channels
    };

    // Tiles from next(row0, col0), one after the other: a tile's first blocks are requested before the results of the one before are worked on
    // (4096 x 2560 -> 2 x 10240 gated by tiles of 128 rows 267 -> 254 us; tiles of 256 x 256 have no registers for it, and plain calls
    // of more tiles than compute units take other forms: ONCE, one tile).
    template <bool ONCE, typename Next>
    static __device__ __forceinline__ void run(const Linear8Args& a, unsigned char* lds, int all_rows, Next&& next_tile)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 31, h = lane >> 5;
        const int wm = wave & 1, wn = wave >> 1;
        const int words = (a.blocks + 3) / 4;
        Source t;
        typedef __attribute__((address_space(3))) void* lds_ptr;
        typedef const __attribute__((address_space(1))) void* global_ptr;
        const auto request = [&](int b, int place, int i) {
            // (gated: the tokens' rows first; the weights' first 4096 x 2560 -> 2 x 10240 with the load behind it takes 224 us instead of 215)
            if constexpr (GATED) i = i < XI ? i + WI : i - XI;
            if (i < WI) {
                const auto wr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w + ((GATED && (i >> 1 & 1) ? (long)a.Cout : 0L) + t.col0) * a.w_ld), 0, t.cols * a.w_ld, 0x00027000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_ptr)(lds + place + XB + (wave + 4 * i) * 1024), 16, t.wo[wo_of(i)], 128 * b, 0, 0);
            } else {
                const auto xr = __builtin_amdgcn_make_buffer_rsrc((void*)(a.x + (long)t.row0 * a.x_ld), 0, t.rows * a.x_ld, 0x00027000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_ptr)(lds + place + (wave + 4 * (i - WI)) * 1024), 16, t.xo[i - WI], 128 * b, 0, 0);
            }
        };
        // scale words, [word of four blocks % 4][BM + BN rows]: a wave requests two groups of 64 rows in turn
        const int sat[2] = {SC + (2 * wave % GROUPS) * 256, SC + ((2 * wave + 1) % GROUPS) * 256};
        const auto request_word = [&](int word, int e) {
            const int w = word < words ? word : words - 1;
            __builtin_amdgcn_global_load_lds((global_ptr)((e ? t.sp[1] : t.sp[0]) + 4 * (long)w), (lds_ptr)(lds + (e ? sat[1] : sat[0]) + (word & 3) * (BM + BN) * 4), 4, 0, 0);
        };
        const auto begin = [&](int row0, int col0) {
            t.row0 = row0;
            t.col0 = col0;
            t.rows = all_rows - row0 < BM ? all_rows - row0 : BM;
            t.cols = a.Cout - col0 < OUT ? a.Cout - col0 : OUT;
            // what a wave requests: 8 rows of 128 bytes at a time, lane l piece (l % 8) ^ (row / 2 % 8) of row l / 8 (rows that are not there: the last one)
            const int piece = ((lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7)) * 16;
            const auto channel = [&](int p) {
                const int c = tile_channel<GATED>(p);
                return c < t.cols ? c : t.cols - 1;
            };
#pragma unroll
            for (int i = 0; i < XI; ++i) {
                const int p = 8 * (wave + 4 * i) + (lane >> 3);
                t.xo[i] = (p < t.rows ? p : t.rows - 1) * a.x_ld + piece;
            }
#pragma unroll
            for (int i = 0; i < WI; ++i)
                if (!GATED || !(i >> 1 & 1)) t.wo[wo_of(i)] = channel(8 * (wave + 4 * i) + (lane >> 3)) * a.w_ld + piece;
#pragma unroll
            for (int i = 0; i < REQ; ++i) request(0, 0, i);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int p = ((2 * wave + e) % GROUPS) * 64 + lane;
                t.sp[e] = p < BM ? a.xs + (long)(row0 + (p < t.rows ? p : t.rows - 1)) * a.xs_ld : a.ws + (long)((GATED && ((p - BM) >> 6 & 1) ? a.Cout : 0) + col0 + channel(p - BM)) * a.ws_ld;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) request_word(e >> 1, e & 1);
#pragma unroll
            for (int b = 1; b < NS; ++b)
                if (b < a.blocks) {
#pragma unroll
                    for (int i = 0; i < REQ; ++i) request(b, b * STAGE, i);
                }
            t.bias = 0.0f;
            const int c = (int)threadIdx.x % OUT;
            if (a.bias && (int)threadIdx.x < BN && c < t.cols) t.bias = a.bias[((int)threadIdx.x < OUT ? 0 : a.Cout) + col0 + c];
        };
        constexpr auto wait = [](int vm, int lgkm) { return (vm & 15) | 0x70 | lgkm << 8 | (vm >> 4) << 14; };
        const auto barrier = [] {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        int row0, col0;
        if (!next_tile(row0, col0)) return;
        begin(row0, col0);
        // the first block and the scale words have come, the others may be on their way
        if (a.blocks >= NS) __builtin_amdgcn_s_waitcnt(wait((NS - 1) * REQ, 0));
        else __builtin_amdgcn_s_waitcnt(wait(0, 0));
        for (;;) {
        barrier();
        f32x16 acc[RT][CT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < CT; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
        // operands: row m of a tile of 32, pieces h and 2 + h of the first half of the block, 4 + h and 6 + h of the second
        const int off = m * 128 + ((h ^ (m >> 1)) & 7) * 16;
        int xb = wm * RT * 4096 + off, wb = XB + wn * CT * 4096 + off, place = 0;
        i32x8 xf[2][RT], wf[2][CT];
        unsigned xs[RT], ws[CT], xn[RT], wn_[CT];
        const auto operand = [&](int at, int tile) {
            return both(*(const i32x4*)(lds + at + tile * 4096), *(const i32x4*)(lds + (at ^ 32) + tile * 4096));
        };
        const auto read_words = [&](int b) {
            const int at = SC + ((b >> 2 & 3) * (BM + BN) + m) * 4;
#pragma unroll
            for (int i = 0; i < RT; ++i) xn[i] = *(const unsigned*)(lds + at + (wm * RT + i) * 128);
#pragma unroll
            for (int j = 0; j < CT; ++j) wn_[j] = *(const unsigned*)(lds + at + BM * 4 + (wn * CT + j) * 128);
        };
#pragma unroll
        for (int j = 0; j < CT; ++j) wf[0][j] = operand(wb, j);
#pragma unroll
        for (int i = 0; i < RT; ++i) xf[0][i] = operand(xb, i);
        read_words(0);
        // MORE: block b + NS exists; NEXT: block b + 1 does
        const auto block = [&](int b, auto more_, auto next_) {
            constexpr bool MORE = decltype(more_)::value, NEXT = decltype(next_)::value;
#pragma unroll
            for (int i = 0; i < RT; ++i) xs[i] = xn[i] >> 8 * (b & 3);
#pragma unroll
            for (int j = 0; j < CT; ++j) ws[j] = wn_[j] >> 8 * (b & 3);
            const int next = NS == 2 ? place ^ STAGE : place + STAGE < SC ? place + STAGE : 0, step = next - place;
            constexpr int issued = PER * (COME - FREE) < REQ ? PER * (COME - FREE) : REQ;
            constexpr int newer = (NS - 2) * REQ + (COME > FREE ? issued + 1 : 0);
#pragma unroll
            for (int n = 0; n < 2 * N; ++n) {
                const int u = n / N, i = n % N / CT, j = n % CT;
                if (NEXT && n == FREE && FREE < COME) {
                    // the block's last reads are done once the barrier is passed
                    __builtin_amdgcn_s_waitcnt(wait(63, 0));
                    barrier();
                }
                if (NEXT && n == COME) {
                    __builtin_amdgcn_s_waitcnt(wait(MORE ? newer : 0, FREE < COME ? 15 : 0));
                    barrier();
                }
                const int first = n < N ? n * READS : NEXT && n >= COME ? (n - COME) * READS : RT + CT;
#pragma unroll
                for (int r = first; r < first + READS && r < RT + CT; ++r) {
                    if (r < CT) wf[n < N][r] = operand(n < N ? wb ^ 64 : wb + step, r);
                    else xf[n < N][r - CT] = operand(n < N ? xb ^ 64 : xb + step, r - CT);
                }
                if (NEXT && n == (COME + READ < 2 * N ? COME + READ : 2 * N - 1)) read_words(b + 1);
                mma(wf[u][j], ws[j], xf[u][i], xs[i], acc[i][j]);
                if (MORE && n >= FREE) {
                    if (n == FREE) request_word((b >> 2) + 2, b & 1);
#pragma unroll
                    for (int e = PER * (n - FREE); e < PER * (n - FREE + 1) && e < REQ; ++e) request(b + NS, place, e);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            xb += step;
            wb += step;
            place = next;
        };
        int b = 0;
        for (; b + NS < a.blocks; ++b) block(b, std::true_type(), std::true_type());
        for (; b + 1 < a.blocks; ++b) block(b, std::false_type(), std::true_type());
        block(b, std::false_type(), std::false_type());
        // (the instruction works on all lanes: nothing of it may move into the branches below)
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < CT; ++j) {
                if constexpr (N == 16) asm volatile("" : "+a"(acc[i][j]));
                else asm volatile("" : "+v"(acc[i][j]));
            }
        // every wave has read its last operands; the bias to where the channels' lanes find it
        if ((int)threadIdx.x < BN) ((float*)(lds + EPI))[threadIdx.x] = t.bias;
        const int r0 = t.row0, c0 = t.col0, rows = t.rows, cols = t.cols;
        __builtin_amdgcn_s_waitcnt(wait(63, 0));
        barrier();
        const bool more = !ONCE && next_tile(row0, col0);
        if (more) begin(row0, col0);
        asm volatile("" ::: "memory");                       // (the requests stay older than the stores below, whose number the wait for them counts on)
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (GATED) gated(a, lds + EPI, acc, r0, c0, rows, cols, lane, wm, wn);
        else if (rows == BM && cols == OUT) plain<true>(a, (const float*)(lds + EPI), acc, r0, c0, rows, cols, m, h, wm, wn);
        else plain<false>(a, (const float*)(lds + EPI), acc, r0, c0, rows, cols, m, h, wm, wn);
        if (!more) return;
        // (the stores above are newer than the next tile's requests: all of a whole tile's, two per 32 rows, may be on their way)
        static_assert(ONCE || GATED, "the stores that the wait counts on");
        constexpr int most = (NS - 1) * REQ + 2 * RT < 63 ? (NS - 1) * REQ + 2 * RT : 63;
        if (a.blocks >= NS && rows == BM && cols == OUT) __builtin_amdgcn_s_waitcnt(wait(most, 0));
        else __builtin_amdgcn_s_waitcnt(wait(0, 0));
        }
    }

    // FULL: every row and channel of the tile is there.
    template <bool FULL>
    static __device__ __forceinline__ void plain(const Linear8Args& a, const float* bias, f32x16 (&acc)[RT][CT], int row0, int col0, int rows, int cols, int m, int h,
                                                 int wm, int wn)
    {
        constexpr int V = Vec16<T>::N, P = 8 / V;            // a lane's runs of 8 channels are P vectors
        constexpr int JS = FULL && RT * CT < 16 ? CT : FULL ? 2 : 1;         // columns of tiles whose base is on its way at a time
        const int c0 = wn * CT * 32 + 8 * h;
        long row[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = (wm * RT + i) * 32 + m;
            row[i] = row0 + (FULL || r < rows ? r : rows - 1);
        }
#pragma unroll
        for (int j0 = 0; j0 < CT; j0 += JS) {
            uint4 g[JS][2][RT][P];
            if (a.base) {
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    const T* base = (const T*)a.base + row[i] * a.base_ld + col0;
#pragma unroll
                    for (int j = 0; j < JS; ++j)
#pragma unroll
                        for (int v = 0; v < 2; ++v)
#pragma unroll
                            for (int w = 0; w < P; ++w) {
                                const int c = c0 + (j0 + j) * 32 + 16 * v + V * w;
                                g[j][v][i][w] = *(const uint4*)(base + (FULL || c < cols ? c : 0));
                            }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            float b8[JS][2][8];
#pragma unroll
            for (int j = 0; j < JS; ++j)
#pragma unroll
                for (int v = 0; v < 2; ++v)
#pragma unroll
                    for (int e = 0; e < 8; ++e) b8[j][v][e] = bias[c0 + (j0 + j) * 32 + 16 * v + e];
            // a row's pieces of a line of memory one after the other (a column of tiles at a time instead: a third more is written than there is,
            // and 4096 x 2560 -> 20480 takes 223 us instead of 208)
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int j = 0; j < JS; ++j)
#pragma unroll
                    for (int v = 0; v < 2; ++v)
#pragma unroll
                        for (int w = 0; w < P; ++w) {
                            const int c = c0 + (j0 + j) * 32 + 16 * v + V * w;
                            float f[V];
#pragma unroll
                            for (int e = 0; e < V; ++e) f[e] = acc[i][j0 + j][8 * v + V * w + e] + b8[j][v][V * w + e];
                            if (a.base) {
                                float o[V];
                                unpack<T>(g[j][v][i][w], o);
#pragma unroll
                                for (int e = 0; e < V; ++e) f[e] += o[e];
                            }
                            if (FULL || ((wm * RT + i) * 32 + m < rows && c < cols)) *(uint4*)((T*)a.y + row[i] * a.y_ld + col0 + c) = pack<T>(f);
                        }
        }
    }

    // acc[i][t] becomes the gated value of tile t and its gates, most[i] the largest magnitude of a lane's row of tile i.
    template <int GATE>
    static __device__ __forceinline__ void gate_values(const float* bias, f32x16 (&acc)[RT][CT], float (&most)[RT], int h, int wn)
    {
#pragma unroll
        for (int i = 0; i < RT; ++i) most[i] = 0.0f;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int v = 0; v < 16; v += 8) {
                const int c = wn * 64 + 32 * h + 16 * t + v;
                float bu[8], bg[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) { bu[e] = bias[c + e]; bg[e] = bias[OUT + c + e]; }
#pragma unroll
                for (int i = 0; i < RT; ++i) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float f = gate_value<GATE>(acc[i][t][v + e] + bu[e], acc[i][t + CT / 2][v + e] + bg[e]);
                        acc[i][t][v + e] = f;
                        most[i] = fmaxf(most[i], fabsf(f));
                    }
                    if constexpr (RT > 1) __builtin_amdgcn_sched_barrier(0);     // (eight chains overlap; more of them do not fit the registers)
                }
            }
        }
    }

    // Tiles 0, 1 of a wave are values, 2, 3 their gates; a block of 128 output channels is the workgroup's, so that a row's scale is the
    // maximum over two waves.
    static __device__ __forceinline__ void gated(const Linear8Args& a, unsigned char* lds, f32x16 (&acc)[RT][CT], int row0, int col0, int rows, int cols, int lane,
                                                 int wm, int wn)
    {
        static_assert(!GATED || CT == 4, "a workgroup has a block of 128 output channels");
        const int m = lane & 31, h = lane >> 5;
        const float* bias = (const float*)lds;               // [128] of values, [128] of gates
        float* top = (float*)lds + BN;                       // [2][BM]
        float most[RT];
        if (cols != OUT) {                                   // channels that are not there (in eights: Cout is a multiple): 0, as is their bias
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int v = 0; v < 16; v += 8)
                    if (wn * 64 + 32 * h + 16 * t + v >= cols)
#pragma unroll
                        for (int i = 0; i < RT; ++i)
#pragma unroll
                            for (int e = 0; e < 8; ++e) acc[i][t][v + e] = acc[i][t + CT / 2][v + e] = 0.0f;
        }
        if (a.gate == SIGE_GATE_GELU) gate_values<SIGE_GATE_GELU>(bias, acc, most, h, wn);
        else gate_values<SIGE_GATE_SILU>(bias, acc, most, h, wn);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            if (most[i] == __uint_as_float(0x7f800000u)) {       // (a NaN is passed over by the maximum, an infinity has to be)
                most[i] = 0.0f;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e) most[i] = fmaxf(most[i], finite_or_0(acc[i][t][e]));
            }
            most[i] = fmaxf(most[i], __shfl_xor(most[i], 32));
            if (h == 0) top[wn * BM + (wm * RT + i) * 32 + m] = most[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = (wm * RT + i) * 32 + m;
            if (r >= rows) continue;
            const int sb = scale_byte(__float_as_uint(fmaxf(most[i], top[(wn ^ 1) * BM + r])));
            const float inv = scale_inverse(sb);
            unsigned char* q = a.q + (long)(row0 + r) * a.q_ld + col0 + wn * 64 + 32 * h;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint4 w;
                w.x = codes4(acc[i][t][0], acc[i][t][1], acc[i][t][2], acc[i][t][3], inv);
                w.y = codes4(acc[i][t][4], acc[i][t][5], acc[i][t][6], acc[i][t][7], inv);
                w.z = codes4(acc[i][t][8], acc[i][t][9], acc[i][t][10], acc[i][t][11], inv);
                w.w = codes4(acc[i][t][12], acc[i][t][13], acc[i][t][14], acc[i][t][15], inv);
                *(uint4*)(q + 16 * t) = w;
            }
            if (wn == 0 && h == 0) {
                unsigned char* s = a.s + (long)(row0 + r) * a.s_ld;
                const int block = col0 / 128, last = (a.Cout - 1) / 128;
                s[block] = (unsigned char)sb;
                if (block == last)
                    for (int e = block + 1; e & 3; ++e) s[e] = 0;
            }
        }
    }
};

// Number t of the my x nx tiles, in strips of five tiles of rows: the workgroups of an XCD, 32 tiles at a time, share both operands in its L2.  (Not in
// eights: rows whose distance is a power of two then ask the same channels of the memory at the same time; gated 4096 x 2560 -> 2 x 10240 by
// tiles of 256 and of 64 rows 220 and 371 us in strips of eight, 211 and 308 in strips of five, 212 and 323 of three.)
__device__ __forceinline__ void tile_place(int t, int nx, int my, int& row, int& col)
{
    constexpr int STRIP = 5;
    const int g = t / (STRIP * nx), rem = t - g * STRIP * nx, high = my - g * STRIP < STRIP ? my - g * STRIP : STRIP;
    col = rem / high;
    row = g * STRIP + rem - col * high;
}

// The workgroup's number among n, so that each XCD (workgroups go to the eight in turn) has a run of them.
__device__ __forceinline__ int xcd_run(int id, int n)
{
    const int per = n / 8, more = n % 8, x = id & 7;
    return x * per + (x < more ? x : more) + (id >> 3);
}

// HALVES: what the last, partial round of tiles over the compute units leaves idle is used by tiles of half the rows, if that takes one round.
template <typename T, bool GATED, int RT, int CT, int NS, int WGS, bool HALVES>
__global__ __launch_bounds__(256, WGS) void rows8_tile_kernel(Linear8Args a)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char tile_lds[];
    using Tile = Tile8<T, GATED, RT, CT, NS>;
    const int rows = rows8_effective(a.rows), id = blockIdx.x;
    const int nx = (a.Cout + Tile::OUT - 1) / Tile::OUT, my = (rows + Tile::BM - 1) / Tile::BM, n = nx * my;
    const int over = n % COMPUTE_UNITS, whole = HALVES && n > COMPUTE_UNITS && over <= COMPUTE_UNITS / 2 ? n - over : n;
    constexpr bool ONCE = HALVES || !GATED;                   // (else the grid is the chip at most, and a workgroup goes from tile to tile)
    if (id < whole) {
        int turn = 0;
        Tile::template run<ONCE>(a, tile_lds, rows, [&](int& row0, int& col0) {
            const int i = id + turn++ * (int)gridDim.x;
            if (i >= whole) return false;
            int row, col;
            tile_place(xcd_run(i, whole), nx, my, row, col);
            row0 = row * Tile::BM;
            col0 = col * Tile::OUT;
            return true;
        });
    } else if constexpr (HALVES) {
        if (id >= whole + 2 * (n - whole)) return;
        const int half = xcd_run(id - whole, 2 * (n - whole));
        int row, col;
        tile_place(whole + half / 2, nx, my, row, col);
        const int first = row * Tile::BM + (half & 1) * (Tile::BM / 2);
        if (first >= rows) return;
        Tile8<T, GATED, RT / 2, CT, NS>::template run<true>(a, tile_lds, rows, [&](int& row0, int& col0) {
            row0 = first;
            col0 = col * Tile::OUT;
            return true;
        });
    }
}

// One launch of the kernel, for an instantiation per file.
template <typename T, bool GATED, int RT, int CT, int NS, int WGS, bool HALVES = false>
inline int launch_tiles(const char* who, const Linear8Args& a, int rows, hipStream_t st)
{
    using Tile = Tile8<T, GATED, RT, CT, NS>;
    const long n = parts_of(a.Cout, Tile::OUT) * parts_of(rows, Tile::BM);
    SIGE_REQUIRE(n < (1L << 23), SIGE_ERR_UNSUPPORTED, "%s: too many rows and channels", who);
    const auto kern = rows8_tile_kernel<T, GATED, RT, CT, NS, WGS, HALVES>;
    if (int rc = allow_lds(who, (const void*)kern, Tile::LDS)) return rc;
    hipLaunchKernelGGL(kern, dim3((unsigned)(HALVES ? n + COMPUTE_UNITS / 2 : !GATED || n < COMPUTE_UNITS ? n : COMPUTE_UNITS)), dim3(256), Tile::LDS, st, a);
    SIGE_LAUNCH_CHECK(who);
    return SIGE_OK;
}

}  // namespace sige
