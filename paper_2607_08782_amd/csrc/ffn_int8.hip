// Grouped SwiGLU expert FFN in 8-bit integers (Sec. II-A of the Director paper: each expert is an
// FFN sub-network), over ragged groups of rows: token rows and weights in 8 bits, a scale for
// each token and each output channel, both products on the integer matrix instructions, whose
// sums are exact (K up to 2^17: 127 x 127 x 2^17 < 2^31).
//
//   1. h = SiLU(a) b,  a, b = (W1 xq, W3 xq) sx sw, in bf16: a row's scale is known only when all of
//      the row is, and h goes to memory and back in between, in half the bytes of fp32.  The
//      rounding, 2^-8 of a value at most, is no more than that to 8 bits, half of 1/127 of the row's
//      largest.
//   2. hq, sh = the rows of h in 8 bits (of one or two tokens by the strips of 3 themselves)
//   3. y = (W2 hq) sh sw; where its strips or tiles are few, by slices of K, whose sums are added
//
// Sums being whole numbers, a row's result is the same bits by whatever kernel and in whatever
// batch.  Rows of codes are padded to whole steps of 128 columns, so no product has a last part of a
// step.  They lie row after row: step after step (128 columns of all rows together), 64 Mixtral-shaped
// tokens took 104 us for 110, and others as long.
#include <algorithm>
#include <type_traits>

#include "int8.h"
#include "stream_tiles.h"

namespace moe {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int STEP = 128;                                // columns (bytes) of a step

struct I8Args {
    const int8_t* w[MOE_MAX_GROUPS];     // per-group weight codes [w_rows][P]
    const float* ws[MOE_MAX_GROUPS];     // and scales [w_rows]
    const int32_t* offsets;              // routed groups' row offsets (device)
    int n_groups, lead, lead_rows;       // lead groups of lead_rows rows come first
    const int8_t* a;                     // row codes [.][P]
    const float* as;                     // and scales
    const int32_t* a_rows;               // row p of the product is row a_rows[p] of a, or p
    int P;                               // bytes of a row of a and of w
    int N;                               // output columns: f (gate/up) or d
    bf16_t* out;                         // h or y
    int64_t pitch;                       // its rows' elements
    uint32_t* most;                      // bits of the largest |h| of a row's blocks [.][blocks]
    int blocks;                          // (of a strip's columns, 16 to 32 of them or a wide one's 64, or of
                                         // half a wave's 32 of a tile)
    const bf16_t* h;                     // down, strips that quantize: h's rows [.][P]
    int K;                               // and their columns
    int32_t* part;                       // split: sums of the slices of K [slices][rows][N]
    int64_t room;                        // sums that part holds
    int32_t* split;                      // and how many slices there are (device)
    int64_t rows;                        // rows of all groups at most
    int slices;                          // strips: slices of K
    int strips;                          // strips a group
    int width;                           // and the output columns of one
    int slots;                           // groups that can hold rows at once
};

// Bits (as a float) of the larger magnitude of two packed bf16 values.
__device__ __forceinline__ uint32_t most_of2(uint32_t w) {
    return max(w << 16 & 0x7fffffffu, w & 0x7fff0000u);
}

// ---------------------------------------------------------------------------
// Strips: groups of few rows, bound by the weight bytes (16 Mixtral-shaped tokens, two experts: gate/up
// 235 MB in 47 us, down 117 MB in 26, of which 5 or more are the start and the end of each).  A workgroup holds 16 TILES weight rows
// of one group (of gate/up half gate rows, half the same up rows) over all of K, its W waves
// taking every W-th step: a weight byte goes from memory to the registers of the one wave that
// multiplies it, and no wave waits for another before the end.  The waves' sums meet in LDS.
// MS: 16-row blocks of token rows held at once
template <int MS, int TILES>
struct StripStep {
    i32x4 b[TILES][2], a[MS][2];
};

constexpr int QUANT_BYTES = 32 * 1024;                    // codes of a strip's rows in LDS, at most

// h's rows row0 .. row0 + n - 1 as codes and scales in LDS, by all threads of a strip: a thread's first
// pieces of a row come while the row's largest magnitude is looked up.
__device__ __forceinline__ void quantize_rows(const I8Args& p, int8_t* codes, float* row_scale, int row0, int n,
                                              int pitch, int tid, int threads) {
    constexpr int HELD = 4;
    const int lane = tid & 63, chunks = p.P / 8;
    __syncthreads();                                     // the last row block's codes are read
    for (int r = 0; r < n; ++r) {
        const bf16_t* const h = p.h + (int64_t)(row0 + r) * p.P;
        const uint32_t* const most = p.most + (int64_t)(row0 + r) * p.blocks;
        Piece<bf16_t, 8> held[HELD];
        auto load = [&](int c0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) held[i].load(h + (int64_t)min(c0 + i * threads, chunks - 1) * 8);
        };
        load(tid);
        uint32_t top = 0;
        for (int b0 = lane; b0 < p.blocks; b0 += 64 * HELD) {
            uint32_t m[HELD];
#pragma unroll
            for (int i = 0; i < HELD; ++i) m[i] = most[min(b0 + 64 * i, p.blocks - 1)];
#pragma unroll
            for (int i = 0; i < HELD; ++i) top = max(top, m[i]);
        }
        const Int8Scale scale(lanes_max(top));
        if (tid == 0) row_scale[r] = scale.s;
#pragma clang loop unroll(disable)
        for (int c0 = tid; c0 < chunks; c0 += HELD * threads) {
            if (c0 != tid) load(c0);
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int c = c0 + i * threads;
                float v[8];
                held[i].values(v);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = c * 8 + e < p.K ? v[e] : 0.f;
                if (c < chunks) scale.template store<true>(v, codes + r * pitch + c * 8);
            }
        }
    }
    __syncthreads();
}

// QUANT (down): p.h's rows, as many as `codes` holds at a time, are quantized as the strip begins, by
// all of its threads, and their scales go to `row_scale`.  SPLIT (down): the strip's slice of K, its
// sums to p.part.
template <bool SWIGLU, int W, int TILES, int MS, int D, bool LONG, bool QUANT = false, bool SPLIT = false>
__device__ __forceinline__ void strip_rows(const I8Args& p, int* red, int g, int n0, int row0, int rows,
                                           int8_t* codes = nullptr, float* row_scale = nullptr,
                                           int slice = 0) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int ROWS = 16 * TILES, LD = ROWS + 4, BM = 16 * MS;
    constexpr int PER_ROW = (SWIGLU ? ROWS / 2 : ROWS) / 4;          // threads of a row's columns
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, quarter = lane >> 4;
    // steps of K, of a slice those of its own
    const int per = SPLIT ? (p.P / STEP + p.slices - 1) / p.slices : 0;
    const int begin = SPLIT ? slice * per : 0, KT = SPLIT ? min(begin + per, p.P / STEP) : p.P / STEP;
    // weight rows of the strip: past the matrix's columns (of the gate half, past its N) they
    // read as zero
    const int valid = max(min(p.width, p.N - n0), 0);
    // the step that a strip of a long K starts with
    const int turn = LONG ? (int)((unsigned)(n0 / p.width) * 3u % (unsigned)(KT - begin)) : 0;
    auto column = [&](int t) { return (t + turn < KT ? t + turn : t + turn - (KT - begin)) * STEP; };
    int boff[TILES];
#pragma unroll
    for (int j = 0; j < TILES; ++j) {
        const int r = (SWIGLU && j >= TILES / 2 ? j - TILES / 2 : j) * 16 + i16;
        boff[j] = r * p.P + quarter * 16;
    }
    const int8_t* const w_lo = p.w[g] + (int64_t)n0 * p.P;
    const int8_t* const w_hi = w_lo + (SWIGLU ? (int64_t)p.N * p.P : 0);
    auto rsrc = [](const void* base, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, bytes, RSRC_WORD3);
    };
    const int block = QUANT ? min(BM, QUANT_BYTES / (p.P + 16)) : BM;
    for (int m0 = 0; m0 < rows; m0 += block) {
        // rows past the group repeat its last one; their sums are not stored
        const int here = min(rows - m0, block), pitch = p.P + 16;    // (the latter: of rows in LDS)
        int a_row[MS];
#pragma unroll
        for (int m = 0; m < MS; ++m) {
            const int r = row0 + min(m0 + 16 * m + i16, rows - 1);
            a_row[m] = !QUANT && p.a_rows ? p.a_rows[r] : r;
        }
        i32x4 acc[MS][TILES];
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j) acc[m][j] = i32x4{0, 0, 0, 0};
        const int8_t* at[MS];
        // past the end of K: no traffic of the weights, and the last step's rows again
        auto load_b = [&](StripStep<MS, TILES>& s, int t) {
            const int at_k = column(t), bytes = t < KT ? valid * p.P - at_k : 0;
            const auto lo = rsrc(w_lo + at_k, bytes), hi = rsrc(w_hi + at_k, bytes);
#pragma unroll
            for (int j = 0; j < TILES; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    s.b[j][u] = __builtin_bit_cast(
                        i32x4, __builtin_amdgcn_raw_buffer_load_b128(SWIGLU && j >= TILES / 2 ? hi : lo,
                                                                     boff[j], 64 * u, 0));
        };
        auto load_a = [&](StripStep<MS, TILES>& s, int t) {
            const int ta = column(min(t, KT - 1));
#pragma unroll
            for (int m = 0; m < MS; ++m)
#pragma unroll
                for (int u = 0; u < 2; ++u) s.a[m][u] = *(const i32x4*)(at[m] + ta + 64 * u);
        };
        // the weights are the matrix instruction's first operand: a lane then holds four
        // consecutive output columns of one row
        auto multiply = [&](const StripStep<MS, TILES>& s) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < TILES; ++j)
#pragma unroll
                    for (int m = 0; m < MS; ++m)
                        acc[m][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(s.b[j][u], s.a[m][u], acc[m][j], 0, 0, 0);
        };
        StripStep<MS, TILES> s[D];
#pragma unroll
        for (int i = 0; i < D; ++i) load_b(s[i], begin + wave + i * W);
#pragma unroll
        for (int m = 0; m < MS; ++m)
            at[m] = QUANT ? codes + min(i16, here - 1) * pitch + quarter * 16
                          : p.a + (int64_t)a_row[m] * p.P + quarter * 16;
        if constexpr (QUANT) quantize_rows(p, codes, row_scale, row0 + m0, here, pitch, tid, 64 * W);
#pragma unroll
        for (int i = 0; i < D; ++i) load_a(s[i], begin + wave + i * W);
        for (int t = begin + wave; t < KT; t += D * W)
#pragma unroll
            for (int i = 0; i < D; ++i) {
                // (past the end: zero weights)
                multiply(s[i]);
                load_b(s[i], t + (i + D) * W);
                load_a(s[i], t + (i + D) * W);
            }

        __syncthreads();                                 // the last row block's sums are read
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j)
                *(i32x4*)&red[(wave * BM + 16 * m + i16) * LD + 16 * j + 4 * quarter] = acc[m][j];
        __syncthreads();
        // four output columns a thread
        for (int i = tid; i < BM * PER_ROW; i += 64 * W) {
            const int r = i / PER_ROW, c = (i % PER_ROW) * 4;
            const bool live = r < here && c < valid;
            const int row = row0 + min(m0 + r, rows - 1);
            if constexpr (SPLIT) {
                i32x4 v = *(const i32x4*)&red[r * LD + c];
#pragma unroll
                for (int q = 1; q < W; ++q) v += *(const i32x4*)&red[(q * BM + r) * LD + c];
                if (live) *(i32x4*)(p.part + (slice * (int64_t)first_row(p, p.n_groups) + row) * p.N + n0 + c) = v;
                continue;
            }
            const float sx = QUANT ? row_scale[min(r, here - 1)] : p.as[p.a_rows ? p.a_rows[row] : row];
            // the sums of a column block at their scales; columns past N: some scale
            auto sum = [&](int col, int first, float (&out)[4]) {
                i32x4 v = *(const i32x4*)&red[r * LD + col];
#pragma unroll
                for (int q = 1; q < W; ++q) v += *(const i32x4*)&red[(q * BM + r) * LD + col];
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = (float)v[e] * sx * p.ws[g][first + min(n0 + c + e, p.N - 1)];
            };
            float y[4];
            sum(c, 0, y);
            if (SWIGLU) {
                float b[4];
                sum(ROWS / 2 + c, p.N, b);
                silu(y);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = c + e < valid ? y[e] * b[e] : 0.f;
            }
            const uint2 w = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
            // (h's rows have room past N)
            if (live) *(uint2*)(p.out + row * p.pitch + n0 + c) = w;
            if (SWIGLU) {
                // the strip's columns of the row are the PER_ROW lanes side by side
                uint32_t most = max(most_of2(w.x), most_of2(w.y));
#pragma unroll
                for (int o = 1; o < PER_ROW; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o, 64));
                if (c == 0 && live) p.most[(int64_t)row * p.blocks + n0 / p.width] = most;
            }
        }
    }
#endif
}

// MAX_MS = 1, 2: no group holds more than 16, 32 rows.  Otherwise each group takes the row blocks it needs (of four,
// two or one alone, 64 Mixtral-shaped tokens take 101.4 us for 100.4, 64 of DeepSeek-V2-Lite 91.6 for 90.1).
template <bool SWIGLU, int W, int TILES, int MAX_MS, int D, bool LONG, bool QUANT, bool SPLIT>
__global__ __launch_bounds__(64 * W, 2) void strip_int8_kernel(I8Args p) {
    constexpr int SUMS = W * 16 * MAX_MS * (16 * TILES + 4);
    static_assert(SUMS * 4 <= 80 * 1024, "two workgroups share a CU's LDS");
    __shared__ __attribute__((aligned(16))) int red[SUMS];
    __shared__ __attribute__((aligned(16))) int8_t codes[QUANT ? QUANT_BYTES : 16];
    __shared__ float row_scale[16];
    const int of_group = SPLIT ? p.strips * p.slices : p.strips, slot = blockIdx.x / of_group;
    const int strip = (int)blockIdx.x - slot * of_group, slice = SPLIT ? strip / p.strips : 0;
    const int n0 = (strip - slice * p.strips) * p.width;
    if (SPLIT && blockIdx.x == 0 && threadIdx.x == 0) *p.split = p.slices;
    Group of;
    if (p.slots < p.n_groups) {
        of = nth_group(p, slot);
    } else {
        of.g = slot;
        of.row0 = __builtin_amdgcn_readfirstlane(first_row(p, slot));
        of.rows = __builtin_amdgcn_readfirstlane(first_row(p, slot + 1)) - of.row0;
    }
    if (of.rows <= 0) return;
    if constexpr (QUANT) {
        strip_rows<SWIGLU, W, TILES, 1, D, LONG, true>(p, red, of.g, n0, of.row0, of.rows, codes, row_scale);
    } else {
        auto rows = [&](auto blocks) {
            strip_rows<SWIGLU, W, TILES, decltype(blocks)::value, D, LONG, false, SPLIT>(
                p, red, of.g, n0, of.row0, of.rows, nullptr, nullptr, slice);
        };
        if (MAX_MS == 1 || of.rows <= 16) {
            rows(std::integral_constant<int, 1>{});
        } else if constexpr (MAX_MS > 1) {
            if (MAX_MS == 2 || of.rows <= 32) rows(std::integral_constant<int, 2>{});
            else if constexpr (MAX_MS > 2) {
                if (of.rows <= 48) rows(std::integral_constant<int, 3>{});
                else rows(std::integral_constant<int, 4>{});
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Wide strips: groups of some rows over a long K.  A workgroup's four waves each hold 16 columns (of
// gate/up 16 gate and the same 16 up rows) over all of K, or a slice of it, and share the token rows:
// these come by direct loads into a ring of RING steps in LDS, once for four waves' weights, while
// as many steps of weights are on their way to each wave's registers.  (Strips whose waves share K read
// every row from the L2 for 32 columns: of 64 Mixtral-shaped tokens' gate/up 58 us, without their rows'
// loads 49, these 49; down 32, 25 and 27.)  One barrier a step; no sums to join.  A step's rows of 128
// bytes hold chunk c of row r at c ^ (r & 7).
//
// 64 Mixtral-shaped tokens: gate/up 235 MB in 50 us, down 117 MB in 28, 4.7 and 4.2 TB/s, of which about 7
// each are the start and the end.
constexpr int WIDE_COLS = 64, WIDE_LDS = 64 * 1024;

template <bool SWIGLU, int MS>
struct WideStrip {
    static constexpr int TILES = SWIGLU ? 2 : 1, LB = 2 * TILES;               // weight loads of a wave's step
    static constexpr int ROWS = MS <= 4 ? 64 : 128, STAGE = ROWS * STEP, LA = ROWS / 32;      // and rows'
    static constexpr int RING = WIDE_LDS / STAGE, AHEAD = RING;
    // behind a step's rows at the time they are waited for: its step's weights, RING - 2 steps
    static constexpr int BEHIND = LB + (RING - 2) * (LA + LB);
    static_assert(BEHIND < 64, "what a wait can count");
};

template <bool SWIGLU, int MS, bool SPLIT>
__device__ __forceinline__ void wide_rows(const I8Args& p, char* ring, int g, int n_first, int row0, int rows,
                                          int slice) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef WideStrip<SWIGLU, MS> S;
    constexpr int TILES = S::TILES;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, quarter = lane >> 4, n0 = n_first + 16 * wave;
    const int per = SPLIT ? (p.P / STEP + p.slices - 1) / p.slices : 0;
    const int begin = SPLIT ? slice * per : 0, KT = (SPLIT ? min(begin + per, p.P / STEP) : p.P / STEP) - begin;
    const int turn = (int)((unsigned)(n_first / WIDE_COLS) * 3u % (unsigned)KT);
    // column of step t; t < KT
    auto column = [&](int t) { return (begin + (t + turn < KT ? t + turn : t + turn - KT)) * STEP; };
    const int valid = max(min(16, p.N - n0), 0);
    const int boff = i16 * p.P + quarter * 16;
    const int8_t* const w_lo = p.w[g] + (int64_t)n0 * p.P;
    const int8_t* const w_hi = w_lo + (SWIGLU ? (int64_t)p.N * p.P : 0);
    auto rsrc = [](const void* base, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, bytes, RSRC_WORD3);
    };
    for (int m0 = 0; m0 < rows; m0 += S::ROWS) {
        const __amdgpu_buffer_rsrc_t ra = rsrc(p.a + (p.a_rows ? 0 : (int64_t)(row0 + m0) * p.P), -1);
        // rows past the group repeat its last one; their sums are not stored
        int aoff[S::LA];
#pragma unroll
        for (int i = 0; i < S::LA; ++i) {
            const int r = min(32 * i + 8 * wave + (lane >> 3), rows - 1 - m0);
            aoff[i] = (p.a_rows ? p.a_rows[row0 + m0 + r] : r) * p.P + ((lane & 7) ^ (lane >> 3)) * 16;
        }
        i32x4 acc[MS][TILES], b[S::AHEAD][TILES][2];
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j) acc[m][j] = i32x4{0, 0, 0, 0};
        // past the end of K, and of a wave whose columns all lie past N: no traffic of the weights; the
        // last step's rows again
        auto load_b = [&](i32x4 (&to)[TILES][2], int t) {
            const int at_k = column(min(t, KT - 1)), bytes = t < KT ? max(valid * p.P - at_k, 0) : 0;
            const auto lo = rsrc(w_lo + at_k, bytes), hi = rsrc(w_hi + at_k, bytes);
#pragma unroll
            for (int j = 0; j < TILES; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    to[j][u] = __builtin_bit_cast(
                        i32x4, __builtin_amdgcn_raw_buffer_load_b128(j > 0 ? hi : lo, boff, 64 * u, 0));
        };
        auto load_a = [&](char* st, int t) {
            const int at_k = column(min(t, KT - 1));
#pragma unroll
            for (int i = 0; i < S::LA; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_void*)(st + (32 * i + 8 * wave) * STEP), 16, aoff[i],
                                                         at_k, 0, 0);
        };
        // In the order of the steps below, which the waits count on: the barriers between them keep the
        // compiler from another.
#pragma unroll
        for (int t = 0; t < S::AHEAD; ++t) {
            const int rows_of = t - (S::AHEAD - (S::RING - 1));
            if (rows_of >= 0) load_a(ring + rows_of * S::STAGE, rows_of);
            __builtin_amdgcn_sched_barrier(0);
            load_b(b[t], t);
            __builtin_amdgcn_sched_barrier(0);
        }
        unsigned here = 0, fill = (S::RING - 1) * S::STAGE;
#pragma clang loop unroll(disable)
        for (int t0 = 0; t0 < KT; t0 += S::AHEAD) {
            // (past the end of K: zero weights.  A way out between the steps would have the compiler wait for
            // every load)
#pragma unroll
            for (int i = 0; i < S::AHEAD; ++i) {
                const int t = t0 + i;
                wait_vm<S::BEHIND>();
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
                // every wave holds the last step's rows in registers: its slot is free
                load_a(ring + fill, t + S::RING - 1);
                __builtin_amdgcn_sched_barrier(0);
                const char* const st = ring + here;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    i32x4 a[MS];
#pragma unroll
                    for (int m = 0; m < MS; ++m)
                        a[m] = *(const i32x4*)(st + (16 * m + i16) * STEP + (((4 * u + quarter) ^ (i16 & 7)) * 16));
#pragma unroll
                    for (int j = 0; j < TILES; ++j)
#pragma unroll
                        for (int m = 0; m < MS; ++m)
                            acc[m][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[i][j][u], a[m], acc[m][j], 0, 0, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                load_b(b[i], t + S::AHEAD);
                __builtin_amdgcn_sched_barrier(0);
                fill = here;
                here = here == (S::RING - 1) * S::STAGE ? 0 : here + S::STAGE;
            }
        }
        wait_vm<0>();                                    // the ring is written no more
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        // four columns of a row a lane
        const int c = n0 + 4 * quarter;
        uint32_t* const s_most = (uint32_t*)ring;        // [waves][ROWS]
#pragma unroll
        for (int m = 0; m < MS; ++m) {
            const int r = m0 + 16 * m + i16, row = row0 + min(r, rows - 1);
            const bool live = r < rows && c < p.N;
            if constexpr (SPLIT) {
                if (live) *(i32x4*)(p.part + (slice * (int64_t)first_row(p, p.n_groups) + row) * p.N + c) = acc[m][0];
                continue;
            }
            const float sx = p.as[p.a_rows ? p.a_rows[row] : row];
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (float)acc[m][0][e] * sx * p.ws[g][min(c + e, p.N - 1)];
            if constexpr (SWIGLU) {
                silu(y);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[e] = c + e < p.N ? y[e] * ((float)acc[m][1][e] * sx * p.ws[g][p.N + min(c + e, p.N - 1)]) : 0.f;
            }
            const uint2 w = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
            // (h's rows have room past N)
            if (live) *(uint2*)(p.out + row * p.pitch + c) = w;
            if (SWIGLU) {
                uint32_t most = max(most_of2(w.x), most_of2(w.y));
                most = max(most, (uint32_t)__shfl_xor((int)most, 16, 64));
                most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
                if (quarter == 0) s_most[wave * S::ROWS + 16 * m + i16] = most;
            }
        }
        if constexpr (SWIGLU) {                          // a strip is a block
            __syncthreads();
            if (tid < 16 * MS && m0 + tid < rows) {
                uint32_t most = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) most = max(most, s_most[q * S::ROWS + tid]);
                p.most[(int64_t)(row0 + m0 + tid) * p.blocks + n_first / WIDE_COLS] = most;
            }
            __syncthreads();                             // the ring may be written again
        }
    }
#endif
}

template <bool SWIGLU, bool SPLIT>
__global__ __launch_bounds__(256, 2) void wide_strip_int8_kernel(I8Args p) {
    __shared__ __attribute__((aligned(1024))) char ring[WIDE_LDS];
    const int of_group = SPLIT ? p.strips * p.slices : p.strips, slot = blockIdx.x / of_group;
    const int strip = (int)blockIdx.x - slot * of_group, slice = SPLIT ? strip / p.strips : 0;
    const int n0 = (strip - slice * p.strips) * WIDE_COLS;
    if (SPLIT && blockIdx.x == 0 && threadIdx.x == 0) *p.split = p.slices;
    Group of;
    if (p.slots < p.n_groups) {
        of = nth_group(p, slot);
    } else {
        of.g = slot;
        of.row0 = __builtin_amdgcn_readfirstlane(first_row(p, slot));
        of.rows = __builtin_amdgcn_readfirstlane(first_row(p, slot + 1)) - of.row0;
    }
    if (of.rows <= 0) return;
    auto rows = [&](auto blocks) {
        wide_rows<SWIGLU, decltype(blocks)::value, SPLIT>(p, ring, of.g, n0, of.row0, of.rows, slice);
    };
    if (of.rows <= 16) rows(std::integral_constant<int, 1>{});
    else if (of.rows <= 32) rows(std::integral_constant<int, 2>{});
    else if (of.rows <= 48) rows(std::integral_constant<int, 3>{});
    else if (of.rows <= 64) rows(std::integral_constant<int, 4>{});
    else if (of.rows <= 96) rows(std::integral_constant<int, 6>{});
    else rows(std::integral_constant<int, 8>{});
}

// ---------------------------------------------------------------------------
// Tiles: groups of many rows, bound by the matrix rate.  A persistent grid of workgroups of
// WM x 2 waves, each TM x TN accumulator tiles of v_mfma_i32_32x32x32_i8: 256 x 256 by eight waves
// (two a SIMD) or, for few tiles, 128 x 128 by four (two workgroups a CU).
//
// Both operands go straight from memory into a ring of RING steps of 64 columns in LDS: a step's
// loads have RING - 2 to RING - 1 steps of products to arrive.  The steps of all of a workgroup's
// tiles are one stream: loads run ahead of the products whatever tile these belong to, so a tile
// starts without waiting for its first operands.  One barrier per step, in its middle: there every
// wave holds its second half's fragments in registers, so the step's ring slot is free, and the next
// step has landed, so the fragments of its first half are read during the second half's products.
//
// LDS rows are 64 bytes; 16-byte chunk c of row r sits at c ^ ((r >> 2) & 3), free of bank conflicts
// for the reads of 32 rows.  The weights are the instruction's first operand, laid out in LDS so that
// a lane's sixteen accumulators are sixteen consecutive output columns of one token row (w_order).  A
// tile's scales come into LDS like its operands, ahead of its first step.
//
// 4096 Mixtral-shaped tokens (3254 rows of two experts): gate/up 415 us (least of twelve 391), down 195
// (177), 1.8 and 2.0 POP/s, near a library's product of such a shape (1.9 to 2.15); the matrix units are busy
// 52 % of the clocks, and the clock falls to 1.8 and 2.0 GHz under the power limit.  Not kept: 128 x 128 a wave, four waves
// (616 -> 677 us), a ring of eight steps with one workgroup a CU for 128 x 128 (even or slower).
constexpr int HALF_LINE = 64;                            // columns (bytes) of a tile's step
constexpr int SCALES = 8;                                // tiles whose scales are kept: the loads' and
                                                         // the products' are RING steps apart, and a
                                                         // tile has two steps at least

// TM x TN accumulator tiles per wave, WM x 2 waves, R steps in the ring
template <int WM, int TM, int TN, int R>
struct TileShape {
    static constexpr int WAVES = 2 * WM, THREADS = 64 * WAVES;
    static constexpr int BM = 32 * WM * TM, BN = 64 * TN;          // token rows, weight rows
    static constexpr int B_CODES = BM * HALF_LINE, STAGE = (BM + BN) * HALF_LINE;
    static constexpr int AT_SX = R * STAGE, AT_SW = AT_SX + SCALES * BM * 4, AT_TOK = AT_SW + SCALES * BN * 4;
    static constexpr int LDS = AT_TOK + 2 * BM * 4;      // the ring, scales, two tiles' token rows
    // direct loads per wave and step: 16 rows each
    static constexpr int AL = BM / 16 / WAVES, BL = BN / 16 / WAVES, LOADS = AL + BL;
    static constexpr int PER_EU = 2;                     // waves a SIMD holds
    static_assert(TM * TN <= 8, "the accumulators of two waves a SIMD");
    static_assert(BM / 64 + BN / 64 == WAVES, "a wave loads 64 scales of a tile");
};

struct I8Tile {
    int row0, valid, n0, slice;
    uint64_t w, ws;                                      // its group's weight codes and scales
};

// Slices of K of a product whose tiles leave workgroups without one: as many, of one, two and four,
// as there are workgroups for, of 2048 columns at least, as far as their sums have room.
constexpr int SLICE_STEPS = 32, MAX_SLICES = 4;

__device__ __forceinline__ int slices_of(int tiles, int steps, int64_t sums, int64_t room) {
    int n = 1;
    while (n < MAX_SLICES && 2 * n * tiles <= (int)gridDim.x && steps >= 2 * n * SLICE_STEPS && 2 * n * sums <= room)
        n *= 2;
    return n;
}

template <bool SWIGLU, int WM, int TM, int TN, int RING, bool SPLIT>
__global__ __launch_bounds__(64 * 2 * WM, 2) void tile_int8_kernel(I8Args p) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef TileShape<WM, TM, TN, RING> S;
    constexpr int BM = S::BM, BN = S::BN, BN_OUT = SWIGLU ? BN / 2 : BN;
    constexpr int AL = S::AL, BL = S::BL, ROUND = 16 * S::WAVES;
    extern __shared__ __attribute__((aligned(1024))) char ring[];
    __shared__ int s_off[MOE_MAX_GROUPS + 1], s_high[MOE_MAX_GROUPS + 1], s_low[MOE_MAX_GROUPS + 1];
    __shared__ I8Tile s_tile[TILE_LIST];
    float* const s_sx = (float*)(ring + S::AT_SX);       // [SCALES][BM]
    float* const s_sw = (float*)(ring + S::AT_SW);       // [SCALES][BN]
    int* const s_tok = (int*)(ring + S::AT_TOK);         // [2][BM]
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2, wn = wave % 2;              // a SIMD's waves hold rows of both halves
    int n_tiles = (p.N + BN_OUT - 1) / BN_OUT;
    const int steps = p.P / HALF_LINE;
    for (int g = tid; g <= p.n_groups; g += S::THREADS) s_off[g] = first_row(p, g);
    __syncthreads();
    if (wave == 0) {
        starts(s_off, p.n_groups, n_tiles, s_high, lane, [](int rows) { return high_tiles<BM>(rows); });
        starts(s_off, p.n_groups, n_tiles, s_low, lane,
               [](int rows) { return (int)ceil_div(rows, BM) - high_tiles<BM>(rows); });
    }
    __syncthreads();
    // few tiles: slices of K, each a column tile of its own
    int slices = 1;
    if constexpr (SPLIT) {
        slices = slices_of(__builtin_amdgcn_readfirstlane(s_high[p.n_groups] + s_low[p.n_groups]), steps,
                           (int64_t)__builtin_amdgcn_readfirstlane(s_off[p.n_groups]) * p.N, p.room);
        if (blockIdx.x == 0 && tid == 0) *p.split = slices;
        if (slices > 1) {
            __syncthreads();
            for (int g = tid; g <= p.n_groups; g += S::THREADS) {
                s_high[g] *= slices;
                s_low[g] *= slices;
            }
            n_tiles *= slices;
            __syncthreads();
        }
    }
    const int per = (steps + slices - 1) / slices;
    const int64_t slice_rows = SPLIT ? __builtin_amdgcn_readfirstlane(s_off[p.n_groups]) : 0;
    const TileShare<BM> tiles(s_off, s_high, s_low, p.n_groups, n_tiles);
    const int n_list = tiles.n_list;                     // this workgroup's tiles
    if (n_list <= 0) return;
    // records of the half of the list that starts with tile q0, half a list ahead of the
    // products' tile (the loads' is RING ahead at most): the half's old ones are used up
    auto list_tiles = [&](int q0) {
        const int q = q0 + tid;
        if (tid >= TILE_LIST / 2 || q >= n_list) return;
        const auto at = tiles.at(q);
        I8Tile t;
        t.w = (uint64_t)p.w[at.g];
        t.ws = (uint64_t)p.ws[at.g];
        t.row0 = at.row0;
        t.valid = at.valid;
        t.slice = SPLIT ? at.n % slices : 0;
        t.n0 = (SPLIT ? at.n / slices : at.n) * BN_OUT;
        s_tile[q % TILE_LIST] = t;
    };
    auto tile_at = [&](int q) {
        I8Tile t = s_tile[q % TILE_LIST];
        t.w = uniform(t.w);
        t.ws = uniform(t.ws);
        t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
        t.valid = __builtin_amdgcn_readfirstlane(t.valid);
        t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
        t.slice = SPLIT ? __builtin_amdgcn_readfirstlane(t.slice) : 0;
        return t;
    };
    auto steps_of = [&](const I8Tile& t) { return SPLIT ? min(per, steps - t.slice * per) : steps; };
    list_tiles(0);
    list_tiles(TILE_LIST / 2);
    __syncthreads();

    // the loads' side of the stream: tile, step of it, operand descriptors, row offsets
    // load i of a wave fills LDS rows ROUND i + 16 wave + lane / 4 of A or B, slot lane % 4
    const int lrow = 16 * wave + (lane >> 2);
    const int lchunk = ((lane & 3) ^ ((lane >> 4) & 3)) * 16;
    auto rsrc = [](uint64_t base) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, -1, RSRC_WORD3);
    };
    __amdgpu_buffer_rsrc_t ra = rsrc(0), rb = ra;
    uint32_t at_k = 0;
    int aoff[AL], boff[BL];
    // gather: the token rows of a tile's rows come into LDS a tile ahead, by a direct load
    // like the ring's (zero past the group)
    auto fetch_tokens = [&](int q) {
        const I8Tile t = tile_at(q);
        if (64 * wave >= BM) return;
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.a_rows + t.row0), (short)0, t.valid * 4, RSRC_WORD3);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(s_tok + (q & 1) * BM + 64 * wave), 4,
                                                 tid * 4, 0, 0, 0);
    };
    if (p.a_rows != nullptr) fetch_tokens(0);
    int lq = -1, left_steps = 0;                         // before the first tile
    auto next_tile = [&]() {
        ++lq;
        const bool live = lq < n_list;
        const I8Tile t = tile_at(live ? lq : n_list - 1);
        if (p.a_rows != nullptr) {
            // Issued a tile ago.  The waits of the loop are for older loads than a step's,
            // but a tile of fewer steps than the ring ends before the first of them.
            if (lq == 0 || steps < RING) {
                wait_vm<0>();
                asm volatile("s_barrier" ::: "memory");
            }
            if (lq + 1 < n_list) fetch_tokens(lq + 1);
        }
        // rows past the group's or the matrix's repeat its last one; past the last tile all lanes
        // are on one row
        auto row_a = [&](int r) {
            return !live ? 0 : p.a_rows != nullptr ? s_tok[(lq & 1) * BM + r] : min(r, t.valid - 1);
        };
        auto row_b = [&](int r) {
            const bool up = SWIGLU && r >= BN / 2;
            return !live ? 0 : min(t.n0 + w_order(up ? r - BN / 2 : r), p.N - 1) + (up ? p.N : 0);
        };
        const int64_t first = p.a_rows != nullptr ? 0 : t.row0;
        ra = rsrc((uint64_t)p.a + first * p.P);
        rb = rsrc(t.w);
#pragma unroll
        for (int i = 0; i < AL; ++i) aoff[i] = row_a(lrow + ROUND * i) * p.P + lchunk;
#pragma unroll
        for (int i = 0; i < BL; ++i) boff[i] = row_b(lrow + ROUND * i) * p.P + lchunk;
        // the tile's scales: its rows' by the first waves, its columns' by the others
        constexpr int ROWS_BY = BM / 64;
        if (live) {
            const int slot = lq & (SCALES - 1);
            if (wave < ROWS_BY) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc((uint64_t)(p.as + first)),
                                                         (lds_void*)(s_sx + slot * BM + 64 * wave), 4,
                                                         row_a(64 * wave + lane) * 4, 0, 0, 0);
            } else {
                const int c = 64 * (wave - ROWS_BY) + lane;
                const bool up = SWIGLU && c >= BN / 2;
                const int col = min(t.n0 + (up ? c - BN / 2 : c), p.N - 1) + (up ? p.N : 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(t.ws),
                                                         (lds_void*)(s_sw + slot * BN + 64 * (wave - ROWS_BY)), 4,
                                                         col * 4, 0, 0, 0);
            }
        }
        at_k = t.slice * per * HALF_LINE;
        left_steps = steps_of(t);
    };
    // direct load i of the stream's next step
    auto load1 = [&](char* st, int i) {
        if (i < AL)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                ra, (lds_void*)(st + (ROUND * i + 16 * wave) * HALF_LINE), 16, aoff[i], at_k, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rb, (lds_void*)(st + S::B_CODES + (ROUND * (i - AL) + 16 * wave) * HALF_LINE), 16, boff[i - AL],
                at_k, 0, 0);
    };
    auto next_step = [&]() {
        --left_steps;
        at_k += HALF_LINE;
    };

    // the products' side: fragment addresses within a step (32-column halves of it by kk)
    const int swz = (r32 >> 2) & 3;
    const int a_row = wm * 32 * TM + r32;
    const int b_row = wn * (SWIGLU ? BN / 4 : BN / 2) + r32;
    auto b_tile = [](int j) { return SWIGLU && j >= TN / 2 ? BN / 2 + (j - TN / 2) * 32 : j * 32; };
    i32x16 acc[TM][TN];                                  // [token tile][weight tile]
    i32x4 fa[2][TM], fb[2][TN];                          // by half of a step
    const int chunk0 = ((0 + half) ^ swz) * 16, chunk1 = ((2 + half) ^ swz) * 16;
    // fragment i of a half of a step: the weights', then the rows'
    auto read1 = [&](const char* st, int kk, int i) {
        st += kk ? chunk1 : chunk0;
        if (i < TN) fb[kk][i] = *(const i32x4*)(st + S::B_CODES + (b_row + b_tile(i)) * HALF_LINE);
        else fa[kk][i - TN] = *(const i32x4*)(st + (a_row + 32 * (i - TN)) * HALF_LINE);
    };
    // the products of a half that follow its read i, behind what was issued before them: the
    // order of reads, loads and products is the source's
    auto multiply = [&](auto half_of, int i) {
        constexpr int KK = decltype(half_of)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = i * TM * TN / (TM + TN); u < (i + 1) * TM * TN / (TM + TN); ++u) {
            const int m = u / TN, j = u % TN;
            acc[m][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[KK][j], fa[KK][m], acc[m][j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // keeps a half's products from being moved past a wait
    auto pin = [&]() {
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(acc[m][j]));
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};

    // a step's loads are issued in two halves of a step of products each: the second of one
    // step, once the slot is free, and the first of the next
    constexpr int EARLY = (S::LOADS + 1) / 2;
    for (int r = 0; r < RING; ++r) {
        char* const st = ring + r * S::STAGE;
        if (left_steps == 0) next_tile();
#pragma unroll
        for (int i = 0; i < EARLY; ++i) load1(st, i);
        if (r == RING - 1) break;
#pragma unroll
        for (int i = EARLY; i < S::LOADS; ++i) load1(st, i);
        next_step();
    }
    wait_vm<(RING - 2) * S::LOADS + EARLY>();
    asm volatile("s_barrier" ::: "memory");
#pragma unroll
    for (int i = 0; i < TM + TN; ++i) read1(ring, 0, i);
    // slots of this step, the next, and the one that loads go to (offsets in the ring)
    unsigned here = 0, next = S::STAGE, fill = (RING - 1) * S::STAGE;
    auto turn = [&]() {                                  // the step's slot is free
        fill = here;
        here = next;
        next = next == (RING - 1) * S::STAGE ? 0 : next + S::STAGE;
    };
    // stores of an epilogue: newer than the loads that the next RING - 2 waits are for
    // (of a split tile there are twice as many: its waits are stricter than they need be)
    constexpr int STORES = SWIGLU ? TM * TN / 2 * 3 : 2 * TM * TN;
    int fresh = 0;
    // the next step has landed: outstanding may be the ones after it, and stores
    auto landed = [&]() {
        if (fresh > 0) {
            wait_vm<(RING - 2) * S::LOADS + STORES>();
            --fresh;
        } else {
            wait_vm<(RING - 2) * S::LOADS>();
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    for (int q = 0; q < n_list; ++q) {
        const I8Tile cur = tile_at(q);
        const int KT = steps_of(cur);
        if (q > 0 && q % (TILE_LIST / 2) == 0) list_tiles(q + TILE_LIST / 2);
        if (wm * 32 * TM >= cur.valid) {                 // no row of this wave's: its loads only
#pragma clang loop unroll(disable)
            for (int t = 0; t < KT; ++t) {
#pragma unroll
                for (int i = EARLY; i < S::LOADS; ++i) load1(ring + fill, i);
                next_step();
                landed();
                turn();
                if (left_steps == 0) next_tile();
#pragma unroll
                for (int i = 0; i < EARLY; ++i) load1(ring + fill, i);
            }
#pragma unroll
            for (int i = 0; i < TM + TN; ++i) read1(ring + here, 0, i);
            continue;
        }
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[m][j][e] = 0;
#pragma clang loop unroll(disable)
        for (int t = 0; t < KT; ++t) {
#pragma unroll
            for (int i = 0; i < TM + TN; ++i) {
                if (2 * i < TM + TN) {
                    read1(ring + here, 1, 2 * i);
                    read1(ring + here, 1, 2 * i + 1);
                }
                if (i >= TM + TN - (S::LOADS - EARLY)) load1(ring + fill, S::LOADS - (TM + TN) + i);
                multiply(first, i);
            }
            pin();
            next_step();
            landed();
            turn();
            if (left_steps == 0) next_tile();
#pragma unroll
            for (int i = 0; i < TM + TN; ++i) {
                if (2 * i < TM + TN) {
                    read1(ring + here, 0, 2 * i);
                    read1(ring + here, 0, 2 * i + 1);
                }
                if (i >= TM + TN - EARLY) load1(ring + fill, i - (TM + TN - EARLY));
                multiply(second, i);
            }
            pin();
        }
        fresh = RING - 2;

        // Every store is issued, those past the group's rows or the output's columns dropped
        // by the descriptor: the waits above count them.
        const int lr = wm * 32 * TM + r32, slot = q & (SCALES - 1);
        if (SPLIT && slices > 1) {
            const __amdgpu_buffer_rsrc_t rp = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(p.part + (cur.slice * slice_rows + cur.row0) * p.N), (short)0, cur.valid * p.N * 4, RSRC_WORD3);
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const int col = cur.n0 + wn * (BN / 2) + 32 * j + 16 * half + e;
                        __builtin_amdgcn_raw_buffer_store_b128(
                            u32x4{(uint32_t)acc[m][j][e], (uint32_t)acc[m][j][e + 1], (uint32_t)acc[m][j][e + 2],
                                  (uint32_t)acc[m][j][e + 3]},
                            rp, col < p.N ? ((lr + 32 * m) * p.N + col) * 4 : A_OOB, 0, 0);
                    }
            continue;
        }
        const __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.out + (int64_t)cur.row0 * p.pitch), (short)0, cur.valid * (int)p.pitch * 2, RSRC_WORD3);
        const __amdgpu_buffer_rsrc_t rm = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.most + (int64_t)cur.row0 * p.blocks), (short)0, cur.valid * p.blocks * 4, RSRC_WORD3);
        const int lc = wn * (SWIGLU ? BN / 4 : BN / 2) + 16 * half;        // column in the tile
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            const float sx = s_sx[slot * BM + lr + 32 * m];
#pragma unroll
            for (int j = 0; j < (SWIGLU ? TN / 2 : TN); ++j) {
                const int c = lc + 32 * j;
                const float* sw = s_sw + slot * BN + c;
                float v[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = (float)acc[m][j][e] * sx * sw[e];
                if constexpr (SWIGLU) {
                    silu(v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] *= (float)acc[m][TN / 2 + j][e] * sx * sw[BN / 2 + e];
                    if (cur.n0 + BN_OUT > p.N)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (cur.n0 + c + e >= p.N) v[e] = 0.f;
                }
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                    u32x4 w;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[i] = pack_bf16x2(v[e + 2 * i], v[e + 2 * i + 1]);
                        if (SWIGLU) most = max(most, most_of2(w[i]));
                    }
                    const int col = cur.n0 + c + e;
                    // (h's rows have room for whole tiles)
                    __builtin_amdgcn_raw_buffer_store_b128(
                        w, ry, SWIGLU || col < p.N ? ((lr + 32 * m) * (int)p.pitch + col) * 2 : A_OOB, 0, 0);
                }
                if (SWIGLU) {
                    most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
                    __builtin_amdgcn_raw_buffer_store_b32(
                        most, rm, half || cur.n0 + c >= p.N ? A_OOB : ((lr + 32 * m) * p.blocks + (cur.n0 + c) / 32) * 4, 0, 0);
                }
            }
        }
    }
#endif
}

// y of the slices' sums: four columns a thread, a workgroup's threads in one row.  64 rows of 4096: 5 us,
// as long as its launch; joined by a strip's last workgroup, whose release writes its XCD's L2 back, the
// FFN takes 114 us in place of 105.
__global__ __launch_bounds__(256) void join_slices_kernel(I8Args p, int64_t first) {
    const int slices = *p.split;
    if (slices == 1) return;                             // the tiles wrote y
    const int wide = (int)ceil_div(p.N, 1024);
    const int64_t total = first_row(p, p.n_groups);
    const int64_t at = first + blockIdx.x, row = at / wide;
    const int c = (int)(at - row * wide) * 1024 + 4 * threadIdx.x;
    // the row's group: the last that starts at or before it
    const int lane = threadIdx.x & 63;
    int g = -1;
    for (int g0 = 0; g0 <= p.n_groups; g0 += 64) {
        const int mine = min(g0 + lane, p.n_groups);
        g += __popcll(__ballot(g0 + lane <= p.n_groups && first_row(p, mine) <= row));
    }
    if (row >= total || c >= p.N) return;
    i32x4 v = *(const i32x4*)(p.part + row * p.N + c);
    for (int q = 1; q < slices; ++q) v += *(const i32x4*)(p.part + (q * total + row) * p.N + c);
    const float* const sw = p.ws[g] + c;
    const float sx = p.as[row];
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (float)v[e] * sx * sw[e];
    *(uint2*)(p.out + row * p.pitch + c) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
}

int launch_join_slices(const I8Args& p, hipStream_t s) {
    return launch_groups(p.rows * ceil_div(p.N, 1024), 256, [&](int64_t first, unsigned n) {
        hipLaunchKernelGGL(join_slices_kernel, dim3(n), dim3(256), 0, s, p, first);
    });
}

template <bool SWIGLU, int WM, int TM, int TN, int RING, bool SPLIT>
int launch_tiles_of(const I8Args& p, hipStream_t s) {
    typedef TileShape<WM, TM, TN, RING> S;
    static LdsGrant grant;
    const int st = allow_dynamic_lds((const void*)tile_int8_kernel<SWIGLU, WM, TM, TN, RING, SPLIT>, S::LDS, grant);
    if (st != MOE_OK) return st;
    const int grid = num_cus() / NUM_XCD * NUM_XCD * (S::PER_EU * 4 / S::WAVES);
    hipLaunchKernelGGL((tile_int8_kernel<SWIGLU, WM, TM, TN, RING, SPLIT>), dim3(grid), dim3(S::THREADS), S::LDS, s, p);
    return launch_status();
}

template <bool SWIGLU, int WM, int TM, int TN, int RING>
int launch_tiles(const I8Args& p, hipStream_t s) {
    if constexpr (!SWIGLU)
        if (p.room > 0) {
            const int st = launch_tiles_of<false, WM, TM, TN, RING, true>(p, s);
            return st != MOE_OK ? st : launch_join_slices(p, s);
        }
    return launch_tiles_of<SWIGLU, WM, TM, TN, RING, false>(p, s);
}

// Whether down strips quantize h's rows themselves: a launch less, but every strip does it again
// (FFN, with the launch and without: one token of DeepSeek-V2-Lite 20.7 and 18.8 us, of
// Qwen3-30B-A3B 10.9 and 9.5; two Mixtral-shaped tokens 60.7 and 59.8; eight tokens 41.0 and 43.2,
// 14.3 and 17.1).
bool strips_quantize(int64_t max_rows, int f) {
    return max_rows <= 2 && max_rows * (int8_cols(f) + 16) <= QUANT_BYTES;
}

// Few rows in a group at most: another shape of a long K's down strips (launch_strips), and gate/up strips
// become as narrow as the rounds of two workgroups a CU allow, so that the last round is as full as the
// others (Mixtral-shaped, 896 strips of 32 columns and 1024 of 28: 16 tokens 73.7 and 71.6 us, 32 tokens
// 90.1 and 88.2; of more rows, which every strip reads, 64 tokens 101.2 and 107.3).
constexpr int64_t FEW_ROWS = 32;

template <bool SWIGLU, int W, int TILES, int D, bool LONG, int MAX_MS = 4>
int launch_strips_of(I8Args& p, int64_t max_rows, hipStream_t s) {
    p.width = 16 * TILES / (SWIGLU ? 2 : 1);
    if (SWIGLU && LONG && max_rows <= FEW_ROWS) {
        const int64_t at_once = 2 * num_cus(), rounds = ceil_div(p.slots * ceil_div(p.N, p.width), at_once);
        while (p.width > 16 && p.slots * ceil_div(p.N, p.width - 4) <= rounds * at_once) p.width -= 4;
    }
    p.strips = (int)ceil_div(p.N, p.width);
    if (SWIGLU) p.blocks = p.strips;                     // a strip is a block
    const dim3 grid((unsigned)(p.slots * p.strips)), block(64 * W);
    const bool few = max_rows <= 16;
    constexpr bool MANY = LONG && !SWIGLU && MAX_MS == 4;    // more than FEW_ROWS
    if constexpr (!SWIGLU && !MANY)
        if (strips_quantize(max_rows, p.K)) {
            hipLaunchKernelGGL((strip_int8_kernel<false, W, TILES, 1, D, LONG, true, false>), grid, block, 0, s, p);
            return launch_status();
        }
    // two slices of K where the strips alone give a CU one workgroup at most (Mixtral-shaped down
    // product, 256 strips of K = 14336: 64 tokens 108 and 105 us)
    constexpr bool SLICED = !SWIGLU && LONG;
    if (SLICED && (int64_t)grid.x <= num_cus() && p.P >= 2 * SLICE_STEPS * HALF_LINE && 2 * p.rows * p.N <= p.room)
        p.slices = 2;
    auto launch = [&](auto split) {
        constexpr bool SPLIT = decltype(split)::value;
        const dim3 all(grid.x * (SPLIT ? p.slices : 1));
        if constexpr (!MANY)
            if (few) {
                hipLaunchKernelGGL((strip_int8_kernel<SWIGLU, W, TILES, 1, D, LONG, false, SPLIT>), all, block, 0, s, p);
                return launch_status();
            }
        hipLaunchKernelGGL((strip_int8_kernel<SWIGLU, W, TILES, MAX_MS, D, LONG, false, SPLIT>), all, block, 0, s, p);
        return launch_status();
    };
    if constexpr (SLICED)
        if (p.slices > 1) {
            const int st = launch(std::true_type{});
            return st != MOE_OK ? st : launch_join_slices(p, s);
        }
    return launch(std::false_type{});
}

template <bool SWIGLU>
int launch_wide_strips(I8Args& p, hipStream_t s) {
    p.strips = (int)ceil_div(p.N, WIDE_COLS);
    if (SWIGLU) p.blocks = p.strips;
    const int64_t groups = (int64_t)p.slots * p.strips;
    if constexpr (!SWIGLU) {
        // slices of K while the strips give a CU one workgroup at most
        while (p.slices < MAX_SLICES && groups * p.slices <= num_cus() &&
               p.P / HALF_LINE >= 2 * p.slices * SLICE_STEPS && 2 * p.slices * p.rows * p.N <= p.room)
            p.slices *= 2;
        if (p.slices > 1) {
            hipLaunchKernelGGL((wide_strip_int8_kernel<false, true>), dim3((unsigned)(groups * p.slices)), dim3(256), 0, s, p);
            const int st = launch_status();
            return st != MOE_OK ? st : launch_join_slices(p, s);
        }
    }
    hipLaunchKernelGGL((wide_strip_int8_kernel<SWIGLU, false>), dim3((unsigned)groups), dim3(256), 0, s, p);
    return launch_status();
}

// A short K gives a strip's waves few steps, and what a strip waits for at its start and end is
// hidden by other workgroups: narrow strips, one step of loads in flight and registers for more
// waves (FFN of 64 tokens, of twice the columns and two steps, of 16 and one: DeepSeek-V2-Lite 97.7 and 91.1 us,
// Qwen3-30B-A3B 22.5 and 20.6).  A long K: 32 columns of gate and up rows, so that token rows are
// read half as often (64 Mixtral-shaped tokens 101.2 us, of 16 columns 111.7), and two steps in flight (4 tokens 57.8,
// one in gate/up 58.6).  Down strips of a long K are few: of 16 columns by eight waves while every strip
// reads few rows (by four waves of 32 columns and by these: 1 token 32.1 and 28.3 us, 4 tokens 57.8 and
// 53.4, 16 tokens 71.6 and 69.0, 32 tokens 88.1 and 87.0, 64 tokens 101.9 and 108.4).  Strips of a long K start
// at other steps of it than their neighbours, and go round: all at the same one, rows of a power of two of
// bytes, they would ask few of the memory's channels at a time (1 token 32.1 and 33.7, 16 tokens 71.6 and
// 75.0, 64 tokens 101.2 and 106.7; a short K is shorter without, 64 DeepSeek-V2-Lite tokens 91.1 and 92.1).
constexpr int SHORT_K = 16 * STEP;

template <bool SWIGLU>
int launch_strips(I8Args& p, int64_t max_rows, hipStream_t s) {
    if (p.P <= SHORT_K) return launch_strips_of<SWIGLU, 4, 2, 1, false>(p, max_rows, s);
    if constexpr (SWIGLU) return launch_strips_of<true, 4, 4, 2, true>(p, max_rows, s);
    else if (max_rows <= FEW_ROWS) return launch_strips_of<false, 8, 1, 2, true, 2>(p, max_rows, s);
    else return launch_strips_of<false, 4, 2, 2, true>(p, max_rows, s);
}

// Wide strips over a long K where a group can hold more than FEW_ROWS rows, up to what one pass over its
// weights takes, and has room for more than 16 on average (FFN, strips or past 64 tokens tiles, and these:
// Mixtral-shaped, 24 tokens 81.6 and 83.6 us, 32 tokens 86.0 and 84.2, 48 tokens 95.3 and 85.3, 64 tokens 100.5
// and 86.8, 96 tokens 106.3 and 91.8, 128 tokens 109.5 and 97.0, 256 tokens 126 and 150; 64 tokens of 8 of 16
// experts of 5120 x 2560, eight rows each, 78.6 and 83.2, 128 tokens 113.8 and 98.1; a short K, 64 tokens of 8
// experts of DeepSeek-V2-Lite, 24.7 and 29.0).
constexpr int64_t WIDE_MAX_ROWS = 128;

// Strips while no group can hold more rows than this, tiles past it (FFN, strips and tiles, without wide ones:
// Mixtral-shaped, 32 tokens 91 and 97 us, 64 tokens 105 and 102, 96 tokens 127 and 105; 64
// DeepSeek-V2-Lite experts, 64 tokens 91 and 97, 128 tokens 125 and 125; Qwen3-30B-A3B, 64 tokens 20
// and 25, 128 tokens 32 and 27).
constexpr int64_t STRIP_MAX_ROWS = 64;

// Tiles of 256 x 256 from this many outputs of a product, of 128 x 128 below, counted over the rows
// that the call has room for (how many there are only the GPU knows).  Gate/up (FFN with 128 x 128
// and 256 x 256, by millions of outputs): 2.2 32 and 39 us, 4.3 163 and 151, 6.3 35.9 and 39.5 but
// 43.8 and 42.2, 17 67 and 60, 23 91 and 79.  Down, K short: 9 42 and 47, 13 42.1 and 47.2, 25 even,
// 34 79 and 75; K long, where slices fill the chip: 1.6 122 and 125, 4.1 176 and 174, 6.4 224 and 202.
constexpr int64_t LARGE_UP = 1 << 22, LARGE_DOWN = 1 << 24, LARGE_SLICED = 1 << 22;

template <bool SWIGLU>
int launch_product(I8Args& p, int64_t max_rows, hipStream_t s) {
    if (p.P > SHORT_K && max_rows > FEW_ROWS && max_rows <= WIDE_MAX_ROWS && p.rows > 16 * (int64_t)p.n_groups)
        return launch_wide_strips<SWIGLU>(p, s);
    if (max_rows <= STRIP_MAX_ROWS) return launch_strips<SWIGLU>(p, max_rows, s);
    if (SWIGLU) p.blocks = (int)ceil_div(p.N, 32);
    const int64_t large = SWIGLU ? LARGE_UP : p.room > 0 ? LARGE_SLICED : LARGE_DOWN;
    return p.rows * p.N >= large ? launch_tiles<SWIGLU, 4, 2, 4, 4>(p, s) : launch_tiles<SWIGLU, 2, 2, 2, 4>(p, s);
}

// ---------------------------------------------------------------------------
// The hidden rows in 8 bits: a row's largest magnitude is that of its blocks', which the first
// product left, so a row needs no pass of its own for it and any number of waves share one: a wave
// takes 64 SEG chunks of eight values.  Bound by the memory rate (3254 rows of 14336: 140 MB in 33 us,
// 4.2 TB/s; 36 with a workgroup for every four units of the rows that there is room for, most of which
// find none), of few rows by its launch (5 us).
template <int SEG>
__global__ __launch_bounds__(256) void quantize_hidden_kernel(const bf16_t* __restrict__ h, int64_t rows,
                                                              int cols, const uint32_t* __restrict__ most,
                                                              int blocks, const int32_t* __restrict__ end,
                                                              int end_base, int units,
                                                              int8_t* __restrict__ q,
                                                              float* __restrict__ scales) {
    const int lane = threadIdx.x & 63;
    const int P = (int)int8_cols(cols), chunks = P / 8;
    const int64_t total = min(rows, (int64_t)end_base + end[0]) * units;
    int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    for (; unit < total; unit += (int64_t)gridDim.x * 4) {
        const int64_t row = unit / units;
        const int part = (int)(unit - row * units);
        Piece<bf16_t, 8> held[SEG];
        auto chunk = [&](int i) { return (part * SEG + i) * 64 + lane; };
#pragma unroll
        for (int i = 0; i < SEG; ++i) held[i].load(h + row * P + (int64_t)min(chunk(i), chunks - 1) * 8);
        uint32_t top = 0;
        for (int b = lane; b < blocks; b += 64) top = max(top, most[row * blocks + b]);
        const Int8Scale scale(lanes_max(top));
        if (part == 0 && lane == 0) scales[row] = scale.s;
#pragma unroll
        for (int i = 0; i < SEG; ++i) {
            const int c = chunk(i);
            float v[8];
            held[i].values(v);
            if (c * 8 + 8 > cols)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c * 8 + j >= cols) v[j] = 0.f;
            if (c < chunks) scale.template store<true>(v, q + row * P + (int64_t)c * 8);
        }
    }
}

int launch_quantize_hidden(const I8Args& p, int64_t rows, int cols, const int32_t* end, int end_base, int8_t* q,
                           float* scales, hipStream_t s) {
    const int64_t lanes = int8_cols(cols) / 8;
    const int seg = rows >= 1024 ? 4 : 1, units = (int)ceil_div(lanes, 64 * seg);
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(rows * units, 4), 8 * num_cus()));
    if (seg == 4)
        hipLaunchKernelGGL(quantize_hidden_kernel<4>, grid, dim3(256), 0, s, p.out, rows, cols, p.most,
                           p.blocks, end, end_base, units, q, scales);
    else
        hipLaunchKernelGGL(quantize_hidden_kernel<1>, grid, dim3(256), 0, s, p.out, rows, cols, p.most,
                           p.blocks, end, end_base, units, q, scales);
    return launch_status();
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// Outputs of a down product from which none is cut into slices: of an eighth of the rows that there
// is room for, 256 x 256 tiles still fill a quarter of the chip.
constexpr int64_t FILLED = 1 << 25;

// workspace: [h in bf16][h codes][h scales][largest |h| of a row's blocks of 16 columns or more]
// [how many slices][sums of slices of K]
struct Layout {
    int64_t hq, hs, most, split, part, room, total;      // room: sums of slices
    Layout(int64_t rows, int d, int f) {
        hq = align256(rows * int8_cols(f) * 2);
        hs = hq + align256(rows * int8_cols(f));
        most = hs + align256(rows * 4);
        split = most + align256(rows * ceil_div(f, 16) * 4);
        part = split + 256;
        // slices where each has SLICE_STEPS and the rows may leave the chip unfilled: as many sums as
        // a tile for every workgroup holds
        room = int8_cols(f) / HALF_LINE >= 2 * SLICE_STEPS && rows * d < FILLED
                   ? std::min<int64_t>(MAX_SLICES * rows * d, 1 << 24) : 0;
        total = part + align256(room * 4);
    }
};

}  // namespace

size_t grouped_ffn_int8_ws_bytes(int64_t rows, int d, int f, int n_groups) {
    return (size_t)Layout(rows, d, f).total + 256;
}

int launch_grouped_ffn_int8(const int8_t* xq, const float* x_scale, int64_t T,
                            const int32_t* row_token, const int32_t* offsets, int n_groups, int lead,
                            int lead_rows, const int8_t* const* w13, const float* const* s13,
                            const int8_t* const* w2, const float* const* s2, int d, int f,
                            int64_t rows, void* y, void* ws, hipStream_t s) {
    if (rows == 0 || T == 0) return MOE_OK;
    const Layout at(rows, d, f);
    char* base = (char*)ws;
    int8_t* hq = (int8_t*)(base + at.hq);
    float* hs = (float*)(base + at.hs);
    // a token reaches an expert at most once
    const int64_t max_rows = row_token ? T : rows;
    I8Args p;
    for (int i = 0; i < MOE_MAX_GROUPS; ++i) {
        p.w[i] = i < n_groups ? w13[i] : nullptr;
        p.ws[i] = i < n_groups ? s13[i] : nullptr;
    }
    p.offsets = offsets;
    p.n_groups = n_groups;
    p.slots = (int)std::min<int64_t>(n_groups, rows);
    p.lead = lead;
    p.slices = 1;
    p.room = 0;
    p.lead_rows = lead_rows;
    p.a = xq;
    p.as = x_scale;
    p.a_rows = row_token;
    p.P = (int)int8_cols(d);
    p.N = f;
    p.out = (bf16_t*)base;
    p.pitch = int8_cols(f);
    p.most = (uint32_t*)(base + at.most);
    p.rows = rows;
    int st = launch_product<true>(p, max_rows, s);
    if (st != MOE_OK) return st;
    p.h = p.out;
    p.K = f;
    if (!strips_quantize(max_rows, f)) {
        st = launch_quantize_hidden(p, rows, f, offsets + n_groups - lead, lead * lead_rows, hq, hs, s);
        if (st != MOE_OK) return st;
    }
    for (int i = 0; i < n_groups; ++i) {
        p.w[i] = w2[i];
        p.ws[i] = s2[i];
    }
    p.a = hq;
    p.as = hs;
    p.a_rows = nullptr;
    p.P = (int)int8_cols(f);
    p.N = d;
    p.out = (bf16_t*)y;
    p.pitch = d;
    p.part = (int32_t*)(base + at.part);
    p.room = at.room;
    p.split = (int32_t*)(base + at.split);
    return launch_product<false>(p, max_rows, s);
}

}  // namespace moe
