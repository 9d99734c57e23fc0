// Grouped SwiGLU expert FFN with 4-bit operands (Sec. II-A of the Director paper: each
// expert is an FFN sub-network), over ragged groups of rows: weights kept in MXFP4, token
// rows and hidden rows quantized to it, both products on the matrix cores' block-scaled
// 4-bit instructions, which take the E8M0 scales as operands.
//
//   0. xq = MXFP4(x), every token once (in few rows, by the strips of 1)
//   1. h = SiLU(W1 xq) * (W3 xq), quantized in the epilogue (a strip or tile of it holds
//      whole blocks of 32 columns, so h is written once, in 4 bits)
//   2. y = W2 h
//
// All operands lie step-major (moe_mxfp4_lay_out): per step of 128 columns, 64 bytes of
// codes a row and then one word of scales a row, rows side by side.  What a product's step
// needs of a row is then no part of a longer line, half of which the cache would fetch for
// nothing (Mixtral-shaped chunk of 777 tokens, the first tiles: 141 us over rows as a matrix
// has them, 125 step-major; 1500 tokens 218 and 190).
#include <algorithm>
#include <type_traits>

#include "mxfp4.h"
#include "stream_tiles.h"

namespace moe {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int STEP_BYTES = 64;                           // codes of a row's 128-column step

struct MxArgs {
    const uint8_t* w[MOE_MAX_GROUPS];    // per-group weight codes [P / 128][rows][64]
    const uint32_t* ws[MOE_MAX_GROUPS];  // and scale words [P / 128][rows]
    const int32_t* offsets;              // routed groups' row offsets (device)
    int n_groups, lead, lead_rows;       // lead groups of lead_rows rows come first
    const uint8_t* a;                    // row codes [P / 128][a_total][64]
    const uint32_t* as;                  // and scale words [P / 128][a_total]
    const int32_t* a_rows;               // row p of the product is row a_rows[p] of a, or p
    int64_t a_total;
    const bf16_t* x;                     // the rows before their quantization [a_total][d]
    int d;
    int KT;                              // 128-column steps of K
    int segment;                         // steps that 32-bit offsets reach
    int N;                               // output columns: f (gate/up) or d
    int w_rows;                          // rows of a weight matrix: 2 f or d
    uint8_t* h;                          // gate/up: hidden codes [hp / 128][h_rows][64]
    uint8_t* hs;                         // and scale words [hp / 128][h_rows], as bytes
    int64_t h_rows;
    int hp;                              // f padded to 128
    bf16_t* y;                           // down: [rows][d]
    int strips;                          // strips a group
    int slots;                           // groups that can hold rows at once
};

__device__ __forceinline__ i32x8 operand(const i32x4& v) {
    return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};    // 4-bit operands use the lower half
}

// SiLU(a) b by the hardware's exponential and reciprocal, an ulp each: h keeps three bits
// of it.  Below a = -88 the reciprocal is zero, and so is h (SiLU is under 2e-36 there).
__device__ __forceinline__ float swiglu(float a, float b) {
    return a * __builtin_amdgcn_rcpf(1.0f + __expf(-a)) * b;
}

// ---------------------------------------------------------------------------
// Strips: groups of few rows, bound by the weight bytes (64 Mixtral-shaped tokens, the FFN of
// two experts: 51 us, 188 MB at 3.7 TB/s; of that gate/up 30 us at 4.2).  A workgroup holds 16 TILES weight
// rows of one group (of gate/up half gate rows, half the same up rows: TILES = 4 makes 32
// hidden columns, one MXFP4 block) over all of K, its W waves taking every W-th step: a
// weight byte goes from memory to the registers of the one wave that multiplies it, and no
// wave waits for another before the end.  The waves' sums meet in LDS, in wave order.
// MS: 16-row blocks of token rows held at once
template <int MS, int TILES, bool QUANT>
struct StripStep {
    i32x4 b[TILES], a[QUANT ? 4 : MS];                   // QUANT: the lane's 32 bf16 values
    uint32_t bs[TILES], as[QUANT ? 1 : MS];
};

// The MXFP4 block of a lane's 32 bf16 values: codes, scale byte.
__device__ __forceinline__ i32x4 mx_block(const i32x4 (&x)[4], uint32_t& byte) {
    float v[4][8];
    uint32_t most = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[u][2 * i] = __uint_as_float((uint32_t)x[u][i] << 16);
            v[u][2 * i + 1] = __uint_as_float((uint32_t)x[u][i] & 0xffff0000u);
        }
        most = max(most, magnitude8(v[u]));
    }
    i32x4 w;
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = (int)mx_encode8(v[u], most, byte);
    return w;
}

// The rows of a group, 16 MS at a time; row0, rows: of the group.  D steps of loads are in
// flight (past the end of K without traffic: every wait counts the same loads).  QUANT (one
// row block): rows come as bf16 values, of which a lane holds just the 32 that are its block
// of the step, and are quantized as they are multiplied.
template <bool SWIGLU, int W, int TILES, int MS, int D, bool QUANT = false>
__device__ __forceinline__ void strip_rows(const MxArgs& p, float* red, int g, int n0, int row0,
                                           int rows) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int ROWS = 16 * TILES, LD = ROWS + 4, BM = 16 * MS;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, quarter = lane >> 4;
    // weight rows of the strip: past the matrix's (or, of the gate half, past its N)
    // columns they read as zero; their scales are some row's
    const int valid = max(min(SWIGLU ? ROWS / 2 : ROWS, p.N - n0), 0);
    int boff[TILES], bsoff[TILES];
#pragma unroll
    for (int j = 0; j < TILES; ++j) {
        const bool up = SWIGLU && j >= TILES / 2;
        const int r = (up ? j - TILES / 2 : j) * 16 + i16;
        boff[j] = r * STEP_BYTES + quarter * 16;
        bsoff[j] = ((up ? p.N : 0) + min(n0 + r, p.N - 1)) * 4;
    }
    auto rsrc = [](const void* base, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, bytes, RSRC_WORD3);
    };
    for (int m0 = 0; m0 < rows; m0 += BM) {
        // rows past the group repeat its last one; their sums are not stored
        int aoff[MS], asoff[MS];
#pragma unroll
        for (int m = 0; m < MS; ++m) {
            const int r = min(m0 + 16 * m + i16, rows - 1);
            const int row = p.a_rows ? p.a_rows[row0 + r] : r;
            aoff[m] = QUANT ? (row * p.d + quarter * 32) * 2 : row * STEP_BYTES + quarter * 16;
            asoff[m] = row * 4;
        }
        const int64_t first = p.a_rows ? 0 : row0;
        const int reach = p.a_rows ? (int)p.a_total : rows;
        f32x4 acc[MS][TILES];
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto load = [&](StripStep<MS, TILES, QUANT>& s, int t) {
            const int live = t < p.KT ? 1 : 0;
            const int64_t brow = (int64_t)t * p.w_rows, arow = t * p.a_total + first;
            const auto lo = rsrc(p.w[g] + (brow + n0) * STEP_BYTES, live * valid * STEP_BYTES);
            const auto hi = rsrc(p.w[g] + (brow + (SWIGLU ? p.N + n0 : n0)) * STEP_BYTES,
                                 live * valid * STEP_BYTES);
            const auto bs = rsrc(p.ws[g] + brow, live * p.w_rows * 4);
            const auto a = QUANT ? rsrc(p.x + first * p.d, live * reach * p.d * 2)
                                 : rsrc(p.a + arow * STEP_BYTES, live * reach * STEP_BYTES);
            const auto as = rsrc(p.as + arow, live * reach * 4);
#pragma unroll
            for (int j = 0; j < TILES; ++j)
                s.b[j] = __builtin_bit_cast(
                    i32x4, __builtin_amdgcn_raw_buffer_load_b128(SWIGLU && j >= TILES / 2 ? hi : lo,
                                                                 boff[j], 0, 0));
#pragma unroll
            for (int j = 0; j < TILES; ++j)
                s.bs[j] = __builtin_amdgcn_raw_buffer_load_b32(bs, bsoff[j], 0, 0);
            if (QUANT) {
#pragma unroll
                for (int u = 0; u < 4; ++u)              // columns past d: zeros
                    s.a[u] = __builtin_bit_cast(
                        i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                   a, 128 * t + 32 * quarter + 8 * u < p.d ? aoff[0] + t * 256 + 16 * u
                                                                           : A_OOB, 0, 0));
                return;
            }
#pragma unroll
            for (int m = 0; m < MS; ++m) {
                s.a[m] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(a, aoff[m], 0, 0));
                s.as[m] = __builtin_amdgcn_raw_buffer_load_b32(as, asoff[m], 0, 0);
            }
        };
        // the weights are the matrix instruction's first operand: a lane then holds four
        // consecutive output columns of one row.  A lane's block of 32 is the word's byte
        // `quarter`
        auto multiply = [&](const StripStep<MS, TILES, QUANT>& s) {
            uint32_t sa[MS];
            i32x4 a[MS];
#pragma unroll
            for (int m = 0; m < MS; ++m) {
                if constexpr (QUANT) {
                    a[m] = mx_block(s.a, sa[m]);
                } else {
                    a[m] = s.a[m];
                    sa[m] = s.as[m] >> (8 * quarter);
                }
            }
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                const uint32_t sb = s.bs[j] >> (8 * quarter);
#pragma unroll
                for (int m = 0; m < MS; ++m)
                    acc[m][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        operand(s.b[j]), operand(a[m]), acc[m][j], 4, 4, 0, (int)sb, 0, (int)sa[m]);
            }
        };
        StripStep<MS, TILES, QUANT> s[D];
#pragma unroll
        for (int i = 0; i < D; ++i) load(s[i], wave + i * W);
        for (int t = wave; t < p.KT; t += D * W)
#pragma unroll
            for (int i = 0; i < D; ++i) {
                multiply(s[i]);
                load(s[i], t + (i + D) * W);
            }

        __syncthreads();                                 // the last row block's sums are read
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j)
                *(f32x4*)&red[(wave * BM + 16 * m + i16) * LD + 16 * j + 4 * quarter] = acc[m][j];
        __syncthreads();
        // four output columns a thread
        constexpr int PER_ROW = (SWIGLU ? ROWS / 2 : ROWS) / 4;
        for (int i = tid; i < BM * PER_ROW; i += 64 * W) {
            const int r = i / PER_ROW, c = (i % PER_ROW) * 4;
            auto sum = [&](int col) {
                f32x4 v = *(const f32x4*)&red[r * LD + col];
#pragma unroll
                for (int q = 1; q < W; ++q) v += *(const f32x4*)&red[(q * BM + r) * LD + col];
                return v;
            };
            const int row = row0 + m0 + r;
            const bool live = m0 + r < rows;
            if (SWIGLU) {
                const f32x4 a = sum(c), b = sum(ROWS / 2 + c);
                float v[4];
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] = swiglu(a[e], b[e]);
                    most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
                }
                // the block is the eight threads of the row
                most = quad_max(most);
                most = max(most, (uint32_t)__shfl_xor((int)most, 4, 64));
                const uint32_t byte = mx_byte(most);
                const float f = mx_factor(byte);
                uint32_t w = 0;
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * f, v[1] * f, 1.0f, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * f, v[3] * f, 1.0f, 1);
                if (byte == 255u) w = 0;
                if (live) {
                    *(uint16_t*)(p.h + ((int64_t)(n0 >> 7) * p.h_rows + row) * STEP_BYTES +
                                 ((n0 & 127) + c) / 2) = (uint16_t)w;
                    if (c == 0)
                        p.hs[((int64_t)(n0 >> 7) * p.h_rows + row) * 4 + ((n0 >> 5) & 3)] =
                            (uint8_t)byte;
                }
            } else if (live && n0 + c < p.N) {
                const f32x4 v = sum(c);
                *(uint2*)(p.y + (int64_t)row * p.N + n0 + c) =
                    make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            }
        }
    }
#endif
}

// Steps of a wave up to which two are in flight, not three or four: more are loads that a
// wave issues before its first product and, past its last step, for nothing (a single token
// through DeepSeek-V2-Lite's experts, whose down product gives a wave 3 steps: 14.8 us with
// four, 13.7 with two; Mixtral's of 28 steps, 16 tokens: 41.8 and 42.5).
constexpr int FEW_STEPS = 6;

// MAX_MS = 1: no group holds more than 16 rows, and the registers of one row block let
// twice the waves in.  Otherwise each group takes the row blocks it needs.
template <bool SWIGLU, int W, int TILES, int MAX_MS, bool QUANT>
__global__ __launch_bounds__(64 * W, QUANT ? 3 : MAX_MS == 1 ? 4 : 2) void strip_mxfp4_kernel(MxArgs p) {
    constexpr int SUMS = W * 16 * MAX_MS * (16 * TILES + 4);
    static_assert(SUMS * 4 <= 80 * 1024, "two workgroups share a CU's LDS");
    __shared__ __attribute__((aligned(16))) float red[SUMS];
    const int slot = blockIdx.x / p.strips;
    const int n0 = ((int)blockIdx.x - slot * p.strips) * 16 * TILES / (SWIGLU ? 2 : 1);
    Group of;
    if (p.slots < p.n_groups) {
        of = nth_group(p, slot);
    } else {
        of.g = slot;
        of.row0 = __builtin_amdgcn_readfirstlane(first_row(p, slot));
        of.rows = __builtin_amdgcn_readfirstlane(first_row(p, slot + 1)) - of.row0;
    }
    if (of.rows <= 0) return;
    // steps of loads in flight that the registers of the row blocks leave room for, four in
    // narrow strips whatever these (128 Mixtral-shaped tokens, whose down product takes them:
    // 75.6 us with three for 33 rows and more, 73.9 so; 64 tokens 51.4 and 50.5)
    constexpr int D = TILES == 4 ? 3 : 4;
    if (QUANT || ((MAX_MS == 1 || of.rows <= 16) && p.KT <= FEW_STEPS * W))
        strip_rows<SWIGLU, W, TILES, 1, 2, QUANT>(p, red, of.g, n0, of.row0, of.rows);
    else if (MAX_MS == 1 || of.rows <= 16)
        strip_rows<SWIGLU, W, TILES, 1, D>(p, red, of.g, n0, of.row0, of.rows);
    else if (of.rows <= 32) strip_rows<SWIGLU, W, TILES, 2, D>(p, red, of.g, n0, of.row0, of.rows);
    else strip_rows<SWIGLU, W, TILES, 4, TILES == 4 ? 2 : 4>(p, red, of.g, n0, of.row0, of.rows);
}

// ---------------------------------------------------------------------------
// Tiles: groups of many rows, bound by the matrix rate.  A persistent grid of workgroups of
// WM x 2 waves, each TM x TN accumulator tiles of v_mfma_scale_f32_32x32x64_f8f6f4: 256 x 256
// by eight waves (two a SIMD) or, for few tiles, 128 x 128 by four (two workgroups a CU).  A
// wave alone on its SIMD keeps 32x32x64 at 6.5 PFLOP/s (random operands, the board's power
// limit) but 16x16x128 only at 4.4: the larger one halves the instructions to issue.
//
// Both operands go straight from memory into a ring of RING steps of 128 columns in LDS,
// the row's codes (64 bytes) and its scale word: a step's loads have RING - 2 to RING - 1
// steps of products to arrive.  The steps of all of a workgroup's tiles are one stream:
// loads run ahead of the products whatever tile these belong to, so a tile starts without
// waiting for its first operands.  One barrier per step, in its middle: there every wave
// holds its second half's fragments in registers, so the step's ring slot is free, and the
// next step has landed, so the fragments of its first half are read during the second
// half's products.  Descriptors stay over a tile and offsets count its steps: with
// descriptors made anew every step the scalar unit issued 120 instructions for 16 products.
//
// LDS rows are 64 bytes; 16-byte chunk c of row r sits at c ^ ((r >> 2) & 3), free of bank
// conflicts for the reads of 32 rows (none counted).  The weights are the instruction's first
// operand; the weight rows of a 32-row block are laid out in LDS so that a lane's sixteen
// accumulators are sixteen consecutive output columns of one token row (w_order): half an
// MXFP4 block of h, or two 16-byte stores of y.
//
// 4096 Mixtral-shaped tokens (3254 rows of two experts): gate/up 206 us, down 100, 3.7 and 3.8
// PFLOP/s; the matrix units are busy 47 and 44 % of the clocks, and the clock falls to 1.9 and
// 2.1 GHz under the power limit: runs with half the scalar instructions, or with a seventh fewer waits, took
// the same time at another clock.
// TM x TN accumulator tiles per wave, WM x 2 waves, R steps in the ring
template <int WM, int TM, int TN, int R>
struct TileShape {
    static constexpr int WAVES = 2 * WM, THREADS = 64 * WAVES;
    static constexpr int BM = 32 * WM * TM, BN = 64 * TN;          // token rows, weight rows
    static constexpr int B_CODES = BM * STEP_BYTES, A_WORDS = (BM + BN) * STEP_BYTES;
    static constexpr int B_WORDS = A_WORDS + BM * 4, STAGE = B_WORDS + BN * 4;
    static constexpr int LDS = R * STAGE + 2 * BM * 4;   // the ring, and two tiles' token rows
    // direct loads per wave and step: 16 rows of codes each, and 64 rows of scale words (of
    // one operand a wave where there are eight, else of both)
    static constexpr int AL = BM / 16 / WAVES, BL = BN / 16 / WAVES, WL = WAVES == 8 ? 1 : 2;
    static constexpr int LOADS = AL + BL + WL;
    static constexpr int PER_EU = 2;                     // waves a SIMD holds
    static_assert(TM * TN <= 8, "the accumulators of two waves a SIMD");
};

struct MxTile {
    int row0, valid, n0;
    uint64_t w, ws;                                      // its group's weight codes and scale words
};

template <bool SWIGLU, int WM, int TM, int TN, int RING>
__global__ __launch_bounds__(64 * 2 * WM, 2) void tile_mxfp4_kernel(MxArgs p) {
#ifdef __HIP_DEVICE_COMPILE__
    typedef TileShape<WM, TM, TN, RING> S;
    constexpr int BM = S::BM, BN = S::BN, BN_OUT = SWIGLU ? BN / 2 : BN;
    constexpr int AL = S::AL, BL = S::BL, ROUND = 16 * S::WAVES;
    extern __shared__ __attribute__((aligned(1024))) char ring[];
    __shared__ int s_off[MOE_MAX_GROUPS + 1], s_high[MOE_MAX_GROUPS + 1], s_low[MOE_MAX_GROUPS + 1];
    __shared__ MxTile s_tile[TILE_LIST];
    int* const s_tok = (int*)(ring + RING * S::STAGE);   // [2][BM]
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / 2, wn = wave % 2;              // a SIMD's waves hold rows of both halves
    // of h, the padding columns too (as zeros)
    const int n_tiles = ((SWIGLU ? p.hp : p.N) + BN_OUT - 1) / BN_OUT;
    for (int g = tid; g <= p.n_groups; g += S::THREADS) s_off[g] = first_row(p, g);
    __syncthreads();
    if (wave == 0) {
        starts(s_off, p.n_groups, n_tiles, s_high, lane, [](int rows) { return high_tiles<BM>(rows); });
        starts(s_off, p.n_groups, n_tiles, s_low, lane,
               [](int rows) { return (int)ceil_div(rows, BM) - high_tiles<BM>(rows); });
    }
    __syncthreads();
    const TileShare<BM> tiles(s_off, s_high, s_low, p.n_groups, n_tiles);
    const int n_list = tiles.n_list;                     // this workgroup's tiles
    if (n_list <= 0) return;
    // records of the half of the list that starts with tile q0, half a list ahead of the
    // products' tile (the loads' is RING ahead at most): the half's old ones are used up
    auto list_tiles = [&](int q0) {
        const int q = q0 + tid;
        if (tid >= TILE_LIST / 2 || q >= n_list) return;
        const auto at = tiles.at(q);
        MxTile t;
        t.w = (uint64_t)p.w[at.g];
        t.ws = (uint64_t)p.ws[at.g];
        t.row0 = at.row0;
        t.valid = at.valid;
        t.n0 = at.n * BN_OUT;
        s_tile[q % TILE_LIST] = t;
    };
    auto tile_at = [&](int q) {
        MxTile t = s_tile[q % TILE_LIST];
        t.w = uniform(t.w);
        t.ws = uniform(t.ws);
        t.row0 = __builtin_amdgcn_readfirstlane(t.row0);
        t.valid = __builtin_amdgcn_readfirstlane(t.valid);
        t.n0 = __builtin_amdgcn_readfirstlane(t.n0);
        return t;
    };
    list_tiles(0);
    list_tiles(TILE_LIST / 2);
    __syncthreads();

    // the loads' side of the stream: tile, step of it, operand descriptors, row offsets
    // load i of a wave fills LDS rows ROUND i + 16 wave + lane / 4 of A or B, slot lane % 4
    const int lrow = 16 * wave + (lane >> 2);
    const int lchunk = ((lane & 3) ^ ((lane >> 4) & 3)) * 16;
    const int a_words = 64 * (wave % (BM / 64)), b_words = 64 * (wave % (BN / 64));
    // word load n: of A's rows or B's
    auto of_a = [&](int n) { return S::WL == 2 ? n == 0 : wave < S::WAVES / 2; };
    // Descriptors stay for up to p.segment steps, which an offset counts; rows past the
    // group's or the matrix's repeat its last one.
    auto rsrc = [](uint64_t base) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, -1, RSRC_WORD3);
    };
    uint64_t base_a = 0, base_b = 0, base_w[S::WL];
    __amdgpu_buffer_rsrc_t ra = rsrc(0), rb = ra, rw[S::WL] = {};
    const uint32_t step_a = (uint32_t)p.a_total * STEP_BYTES, step_b = (uint32_t)p.w_rows * STEP_BYTES;
    uint32_t at_a = 0, at_b = 0, at_w[S::WL], step_w[S::WL];
    int aoff[AL], boff[BL], woff[S::WL], w_lds[S::WL];
#pragma unroll
    for (int n = 0; n < S::WL; ++n) {
        w_lds[n] = of_a(n) ? S::A_WORDS + a_words * 4 : S::B_WORDS + b_words * 4;
        step_w[n] = (of_a(n) ? step_a : step_b) / (STEP_BYTES / 4);
    }
    // gather: the token rows of a tile's rows come into LDS a tile ahead, by a direct load
    // like the ring's (zero past the group)
    auto fetch_tokens = [&](int q) {
        const MxTile t = tile_at(q);
        if (64 * wave >= BM) return;
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.a_rows + t.row0), (short)0, t.valid * 4, RSRC_WORD3);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void*)(s_tok + (q & 1) * BM + 64 * wave), 4,
                                                 tid * 4, 0, 0, 0);
    };
    if (p.a_rows != nullptr) fetch_tokens(0);
    int lq = -1, lkt = 0, left_steps = 0;                // before the first tile
    // the next segment of the tile's steps, or the next tile
    auto next_segment = [&]() {
        if (lkt < p.KT && lq >= 0) {
            base_a += (uint64_t)p.segment * p.a_total * STEP_BYTES;
            base_b += (uint64_t)p.segment * p.w_rows * STEP_BYTES;
#pragma unroll
            for (int n = 0; n < S::WL; ++n)
                base_w[n] += (uint64_t)p.segment * (of_a(n) ? p.a_total : p.w_rows) * 4;
        } else {
            ++lq;
            lkt = 0;
            const bool live = lq < n_list;
            const MxTile t = tile_at(live ? lq : n_list - 1);
            if (p.a_rows != nullptr) {
                // Issued a tile ago.  The waits of the loop are for older loads than a step's,
                // but a tile of fewer steps than the ring ends before the first of them.
                if (lq == 0 || p.KT < RING) {
                    wait_vm<0>();
                    asm volatile("s_barrier" ::: "memory");
                }
                if (lq + 1 < n_list) fetch_tokens(lq + 1);
            }
            // past the last tile: all lanes on one row
            auto row_a = [&](int r) {
                return !live ? 0 : p.a_rows != nullptr ? s_tok[(lq & 1) * BM + r] : min(r, t.valid - 1);
            };
            auto row_b = [&](int r) {
                const bool up = SWIGLU && r >= BN / 2;
                return !live ? 0 : min(t.n0 + w_order(up ? r - BN / 2 : r), p.N - 1) + (up ? p.N : 0);
            };
            const int64_t first = p.a_rows != nullptr ? 0 : t.row0;
            base_a = (uint64_t)p.a + first * STEP_BYTES;
            base_b = t.w;
#pragma unroll
            for (int i = 0; i < AL; ++i) aoff[i] = row_a(lrow + ROUND * i) * STEP_BYTES + lchunk;
#pragma unroll
            for (int i = 0; i < BL; ++i) boff[i] = row_b(lrow + ROUND * i) * STEP_BYTES + lchunk;
#pragma unroll
            for (int n = 0; n < S::WL; ++n) {
                base_w[n] = of_a(n) ? (uint64_t)p.as + first * 4 : t.ws;
                woff[n] = (of_a(n) ? row_a(a_words + lane) : row_b(b_words + lane)) * 4;
            }
        }
        ra = rsrc(base_a), rb = rsrc(base_b);
        at_a = at_b = 0;
#pragma unroll
        for (int n = 0; n < S::WL; ++n) {
            rw[n] = rsrc(base_w[n]);
            at_w[n] = 0;
        }
        left_steps = min(p.segment, p.KT - lkt);
        lkt += left_steps;
    };
    // direct load i of the stream's next step
    auto load1 = [&](char* st, int i) {
        if (i < AL) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                ra, (lds_void*)(st + (ROUND * i + 16 * wave) * STEP_BYTES), 16, aoff[i], at_a, 0, 0);
        } else if (i < AL + BL) {
            const int b = i - AL;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rb, (lds_void*)(st + S::B_CODES + (ROUND * b + 16 * wave) * STEP_BYTES), 16, boff[b], at_b,
                0, 0);
        } else {
            const int n = i - AL - BL;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw[n], (lds_void*)(st + w_lds[n]), 4, woff[n], at_w[n],
                                                     0, 0);
        }
    };
    auto next_step = [&]() {
        --left_steps;
        at_a += step_a, at_b += step_b;
#pragma unroll
        for (int n = 0; n < S::WL; ++n) at_w[n] += step_w[n];
    };

    // the products' side: fragment addresses within a step (16-column halves of it by kk)
    const int swz = (r32 >> 2) & 3;
    const int a_row = wm * 32 * TM + r32;
    const int b_row = wn * (SWIGLU ? BN / 4 : BN / 2) + r32;
    auto b_tile = [](int j) { return SWIGLU && j >= TN / 2 ? BN / 2 + (j - TN / 2) * 32 : j * 32; };
    f32x16 acc[TM][TN];                                  // [token tile][weight tile]
    i32x4 fa[2][TM], fb[2][TN];                          // by half of a step
    int sa[TM], sb[TN], na[TM], nb[TN];                  // scale words, this step's and the next's
    const int chunk0 = ((0 + half) ^ swz) * 16, chunk1 = ((2 + half) ^ swz) * 16;
    // fragment i of a half of a step: the weights', then the rows'
    auto read1 = [&](const char* st, int kk, int i) {
        st += kk ? chunk1 : chunk0;
        if (i < TN) fb[kk][i] = *(const i32x4*)(st + S::B_CODES + (b_row + b_tile(i)) * STEP_BYTES);
        else fa[kk][i - TN] = *(const i32x4*)(st + (a_row + 32 * (i - TN)) * STEP_BYTES);
    };
    auto read_word = [&](const char* st, int i) {
        if (i < TN) nb[i] = *(const int*)(st + S::B_WORDS + (b_row + b_tile(i)) * 4);
        else na[i - TN] = *(const int*)(st + S::A_WORDS + (a_row + 32 * (i - TN)) * 4);
    };
    // blocks `half` and 2 + half of the word are the lane's in the two halves of a step
    auto take_words = [&]() {
#pragma unroll
        for (int j = 0; j < TN; ++j) sb[j] = (int)((uint32_t)nb[j] >> (8 * half));
#pragma unroll
        for (int m = 0; m < TM; ++m) sa[m] = (int)((uint32_t)na[m] >> (8 * half));
    };
    // the products of a half that follow its read i, behind what was issued before them: the
    // order of reads, loads and products is the source's
    auto multiply = [&](auto half_of, int i) {
        constexpr int KK = decltype(half_of)::value;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = i * TM * TN / (TM + TN); u < (i + 1) * TM * TN / (TM + TN); ++u) {
            const int m = u / TN, j = u % TN;
            acc[m][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
                operand(fb[KK][j]), operand(fa[KK][m]), acc[m][j], 4, 4, 2 * KK, sb[j], 2 * KK, sa[m]);
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
        if (left_steps == 0) next_segment();
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
    for (int i = 0; i < TM + TN; ++i) {
        read1(ring, 0, i);
        read_word(ring, i);
    }
    // slots of this step, the next, and the one that loads go to (offsets in the ring)
    unsigned here = 0, next = S::STAGE, fill = (RING - 1) * S::STAGE;
    auto turn = [&]() {                                  // the step's slot is free
        fill = here;
        here = next;
        next = next == (RING - 1) * S::STAGE ? 0 : next + S::STAGE;
    };
    // stores of an epilogue: newer than the loads that the next RING - 2 waits are for
    constexpr int STORES = SWIGLU ? TM * TN / 2 + TM : 2 * TM * TN;
    int fresh = 0;
    // the next step has landed: outstanding may be the two after it, and stores
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
        const MxTile cur = tile_at(q);
        if (q > 0 && q % (TILE_LIST / 2) == 0) list_tiles(q + TILE_LIST / 2);
        if (wm * 32 * TM >= cur.valid) {                 // no row of this wave's: its loads only
#pragma clang loop unroll(disable)
            for (int t = 0; t < p.KT; ++t) {
#pragma unroll
                for (int i = EARLY; i < S::LOADS; ++i) load1(ring + fill, i);
                next_step();
                landed();
                turn();
                if (left_steps == 0) next_segment();
#pragma unroll
                for (int i = 0; i < EARLY; ++i) load1(ring + fill, i);
            }
#pragma unroll
            for (int i = 0; i < TM + TN; ++i) {
                read1(ring + here, 0, i);
                read_word(ring + here, i);
            }
            continue;
        }
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[m][j][e] = 0.f;
#pragma clang loop unroll(disable)
        for (int t = 0; t < p.KT; ++t) {
            take_words();
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
            if (left_steps == 0) next_segment();
#pragma unroll
            for (int i = 0; i < TM + TN; ++i) {
                if (2 * i < TM + TN) {
                    read1(ring + here, 0, 2 * i);
                    read1(ring + here, 0, 2 * i + 1);
                    read_word(ring + here, 2 * i);
                    read_word(ring + here, 2 * i + 1);
                }
                if (i >= TM + TN - EARLY) load1(ring + fill, i - (TM + TN - EARLY));
                multiply(second, i);
            }
            pin();
        }
        fresh = RING - 2;

        // Every store is issued, those past the group's rows or the output's columns dropped
        // by the descriptor: the waits above count them.
        const int lr = wm * 32 * TM + r32;
        if (SWIGLU) {
            const int col = cur.n0 + wn * (BN / 4);
            const __amdgpu_buffer_rsrc_t rh = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(p.h + ((int64_t)(col >> 7) * p.h_rows + cur.row0) * STEP_BYTES), (short)0,
                cur.valid * STEP_BYTES, RSRC_WORD3);
            const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(p.hs + ((int64_t)(col >> 7) * p.h_rows + cur.row0) * 4), (short)0,
                cur.valid * 4, RSRC_WORD3);
#pragma unroll
            for (int m = 0; m < TM; ++m) {
                uint32_t bytes = 0;
#pragma unroll
                for (int j = 0; j < TN / 2; ++j) {
                    float v[16];
                    uint32_t most = 0;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        v[e] = swiglu(acc[m][j][e], acc[m][TN / 2 + j][e]);
                        if (cur.n0 + BN_OUT > p.N && col + 32 * j + 16 * half + e >= p.N) v[e] = 0.f;
                        most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
                    }
                    most = max(most, (uint32_t)__shfl_xor((int)most, 32, 64));
                    uint32_t byte;
                    u32x2 w;
                    w[0] = mx_encode8(v, most, byte);
                    w[1] = mx_encode8(v + 8, most, byte);
                    bytes |= byte << (8 * j);
                    __builtin_amdgcn_raw_buffer_store_b64(
                        w, rh, (lr + 32 * m) * STEP_BYTES + ((col & 127) + 32 * j + 16 * half) / 2, 0, 0);
                }
                const int at = half ? A_OOB : (lr + 32 * m) * 4 + ((col >> 5) & 3);
                if (TN == 4) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)bytes, rs, at, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b8((uint8_t)bytes, rs, at, 0, 0);
            }
        } else {
            const __amdgpu_buffer_rsrc_t ry = __builtin_amdgcn_make_buffer_rsrc(
                (void*)(p.y + (int64_t)cur.row0 * p.N), (short)0, cur.valid * p.N * 2, RSRC_WORD3);
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; e += 8) {
                        const int col = cur.n0 + wn * (BN / 2) + 32 * j + 16 * half + e;
                        u32x4 w;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            w[i] = pack_bf16x2(acc[m][j][e + 2 * i], acc[m][j][e + 2 * i + 1]);
                        __builtin_amdgcn_raw_buffer_store_b128(
                            w, ry, col < p.N ? ((lr + 32 * m) * p.N + col) * 2 : A_OOB, 0, 0);
                    }
        }
    }
#endif
}

template <bool SWIGLU, int WM, int TM, int TN, int RING>
int launch_tiles(const MxArgs& p, int cus, hipStream_t s) {
    typedef TileShape<WM, TM, TN, RING> S;
    static LdsGrant grant;
    const int st = allow_dynamic_lds((const void*)tile_mxfp4_kernel<SWIGLU, WM, TM, TN, RING>, S::LDS, grant);
    if (st != MOE_OK) return st;
    const int grid = cus / NUM_XCD * NUM_XCD * (S::PER_EU * 4 / S::WAVES);
    hipLaunchKernelGGL((tile_mxfp4_kernel<SWIGLU, WM, TM, TN, RING>), dim3(grid), dim3(S::THREADS),
                       S::LDS, s, p);
    return launch_status();
}

// Whether gate/up strips quantize the token rows themselves: a launch less, but every strip
// does it again (FFN, with the launch and without: one token, DeepSeek-V2-Lite 16.5 and
// 14.8 us, Qwen3-30B-A3B 13.9 and 11.2; 16 tokens 34.1 and 33.0, 14.2 and 12.3; Mixtral-shaped,
// twice the steps, 8 tokens 39.2 and 39.0, 16 tokens 40.0 and 41.8).
bool strips_quantize(int64_t max_rows, int d) {
    return max_rows <= 16 && max_rows * (mx_cols(d) / 128) <= 256;
}

template <bool SWIGLU, int W, int TILES>
int launch_strips_of(MxArgs& p, int64_t max_rows, hipStream_t s) {
    p.strips = (int)ceil_div(SWIGLU ? 2 * p.hp : p.N, 16 * TILES);
    const dim3 grid((unsigned)(p.slots * p.strips)), block(64 * W);
    if (SWIGLU && strips_quantize(max_rows, p.d))
        hipLaunchKernelGGL((strip_mxfp4_kernel<SWIGLU, W, TILES, 1, SWIGLU>), grid, block, 0, s, p);
    else if (max_rows <= 16)
        hipLaunchKernelGGL((strip_mxfp4_kernel<SWIGLU, W, TILES, 1, false>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((strip_mxfp4_kernel<SWIGLU, W, TILES, 4, false>), grid, block, 0, s, p);
    return launch_status();
}

// Two waves a strip where there are strips enough to fill the chip (64 DeepSeek-V2-Lite-
// shaped experts, 64 tokens: FFN 63 us with four, 52 with two), else four (Mixtral-shaped
// down product, 64 tokens, 128 strips: 31 us with two, 20 with four), of half the weight
// rows where that still leaves CUs without one (17).
template <bool SWIGLU>
int launch_strips(MxArgs& p, int64_t max_rows, int cus, hipStream_t s) {
    const int64_t n = p.slots * ceil_div(SWIGLU ? 2 * p.hp : p.N, 64);
    if (n >= 4 * cus) return launch_strips_of<SWIGLU, 2, 4>(p, max_rows, s);
    if constexpr (!SWIGLU)
        if (n < 2 * cus) return launch_strips_of<false, 4, 2>(p, max_rows, s);
    return launch_strips_of<SWIGLU, 4, 4>(p, max_rows, s);
}

// Strips while no group can hold more rows than this, tiles past it (FFN, strips and tiles:
// Mixtral-shaped, 40 tokens 47 and 64 us, 96 tokens 67 and 68, 128 tokens 75 and 71, 200 tokens
// 94 and 78; 64 DeepSeek-V2-Lite experts, 128 tokens 63 and 68, 200 tokens 72 and 76; an eighth
// of them, 256 tokens 40 and 22; Qwen3-30B-A3B, 128 tokens 23 and 20).
constexpr int64_t STRIP_MAX_ROWS = 128;

// Tiles of 256 x 256 from this many outputs of a product (a round of them over the chip), of
// 128 x 128 below, counted over the rows that the call has room for: how many there are only
// the GPU knows (FFN, all of one size: Mixtral-shaped, 400 tokens 103 and 87 us, 1500 tokens
// 162 and 194; DeepSeek-V2-Lite on one of eight, 512 tokens 29 and 24, 2048 tokens 38 and 41,
// 8192 tokens 90 and 114.  777 Mixtral-shaped tokens, where the products differ: 124 and 121,
// by the rule 104).
constexpr int64_t LARGE_WORK = (int64_t)256 * 256 * 256;

// steps whose offsets from the first one's stay below 2^31
int segment_steps(int64_t a_rows, int64_t w_rows) {
    return (int)std::max<int64_t>(0x7fffffff / (std::max(a_rows, w_rows) * STEP_BYTES), 1);
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// workspace: [x codes][x scale words][h codes][h scale words], step-major
struct Layout {
    int64_t xs, h, hs, total;
    Layout(int64_t T, int64_t rows, int d, int f) {
        xs = align256(T * mx_cols(d) / 2);
        h = xs + align256(T * mx_cols(d) / 32);
        hs = h + align256(rows * mx_cols(f) / 2);
        total = hs + align256(rows * mx_cols(f) / 32);
    }
};

}  // namespace

size_t grouped_ffn_mxfp4_ws_bytes(int64_t T, int64_t rows, int d, int f) {
    return (size_t)Layout(T, rows, d, f).total + 256;
}

int launch_grouped_ffn_mxfp4(const void* x, int64_t T, const int32_t* row_token,
                             const int32_t* offsets, int n_groups, int lead, int lead_rows,
                             const uint8_t* const* w13, const uint32_t* const* s13,
                             const uint8_t* const* w2, const uint32_t* const* s2, int d, int f,
                             int64_t rows, void* y, void* ws, hipStream_t s) {
    if (rows == 0 || T == 0) return MOE_OK;
    const Layout at(T, rows, d, f);
    char* base = (char*)ws;
    // a token reaches an expert at most once
    const int64_t max_rows = row_token ? T : rows;
    int st = MOE_OK;
    if (!strips_quantize(max_rows, d)) {
        st = launch_quantize_mxfp4_steps((const bf16_t*)x, T, d, (uint8_t*)base,
                                         (uint32_t*)(base + at.xs), s);
        if (st != MOE_OK) return st;
    }
    MxArgs p;
    for (int i = 0; i < MOE_MAX_GROUPS; ++i) {
        p.w[i] = i < n_groups ? w13[i] : nullptr;
        p.ws[i] = i < n_groups ? s13[i] : nullptr;
    }
    p.offsets = offsets;
    p.n_groups = n_groups;
    p.slots = (int)std::min<int64_t>(n_groups, rows);
    p.lead = lead;
    p.lead_rows = lead_rows;
    p.a = (const uint8_t*)base;
    p.as = (const uint32_t*)(base + at.xs);
    p.a_rows = row_token;
    p.a_total = T;
    p.x = (const bf16_t*)x;
    p.d = d;
    p.KT = (int)(mx_cols(d) / 128);
    p.segment = segment_steps(T, 2 * f);
    p.N = f;
    p.w_rows = 2 * f;
    p.h = (uint8_t*)base + at.h;
    p.hs = (uint8_t*)base + at.hs;
    p.h_rows = rows;
    p.hp = (int)mx_cols(f);
    p.y = nullptr;
    const int cus = num_cus();
    st = max_rows <= STRIP_MAX_ROWS ? launch_strips<true>(p, max_rows, cus, s)
         : rows * p.N >= LARGE_WORK   ? launch_tiles<true, 4, 2, 4, 3>(p, cus, s)
                                      : launch_tiles<true, 2, 2, 2, 4>(p, cus, s);
    if (st != MOE_OK) return st;
    for (int i = 0; i < n_groups; ++i) {
        p.w[i] = w2[i];
        p.ws[i] = s2[i];
    }
    p.a = p.h;
    p.as = (const uint32_t*)p.hs;
    p.a_rows = nullptr;
    p.a_total = rows;
    p.KT = p.hp / 128;
    p.segment = segment_steps(rows, d);
    p.N = d;
    p.w_rows = d;
    p.y = (bf16_t*)y;
    return max_rows <= STRIP_MAX_ROWS ? launch_strips<false>(p, max_rows, cus, s)
           : rows * p.N >= LARGE_WORK ? launch_tiles<false, 4, 2, 4, 3>(p, cus, s)
                                      : launch_tiles<false, 2, 2, 2, 4>(p, cus, s);
}

}  // namespace moe
