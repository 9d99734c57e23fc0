// Grouped SwiGLU expert FFN with 4-bit operands (Sec. II-A of the Director paper: each
// expert is an FFN sub-network), over ragged groups of rows: weights kept in MXFP4, token
// rows and hidden rows quantized to it, both products on the matrix cores' block-scaled
// 4-bit instructions, which take the E8M0 scales as operands.
//
//   0. xq = MXFP4(x), every token once
//   1. h = SiLU(W1 xq) * (W3 xq), quantized in the epilogue (a strip or tile of it holds
//      whole blocks of 32 columns, so h is written once, in 4 bits)
//   2. y = W2 h
//
// Scales are kept as words [128-column step][row] (moe_mxfp4_scale_words): the lanes of a
// fragment read them side by side, one word a row and step.
#include "mxfp4.h"

namespace moe {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t RSRC_WORD3 = 0x00020000;              // raw buffer: 32-bit data format
constexpr int STEP_BYTES = 64;                           // codes of a row's 128-column step

struct MxArgs {
    const uint8_t* w[MOE_MAX_GROUPS];    // per-group weight codes [rows][P / 2]
    const uint32_t* ws[MOE_MAX_GROUPS];  // and scale words [P / 128][rows]
    const int32_t* offsets;              // routed groups' row offsets (device)
    int n_groups, lead, lead_rows;       // lead groups of lead_rows rows come first
    const uint8_t* a;                    // row codes [a_total][P / 2]
    const uint32_t* as;                  // and scale words [P / 128][a_total]
    const int32_t* a_rows;               // row p of the product is row a_rows[p] of a, or p
    int64_t a_total;
    int KT;                              // 128-column steps of K
    int N;                               // output columns: f (gate/up) or d
    int w_rows;                          // rows of a weight matrix: 2 f or d
    uint8_t* h;                          // gate/up: hidden codes [h_rows][hp / 2]
    uint8_t* hs;                         // and scale words [hp / 128][h_rows], as bytes
    int64_t h_rows;
    int hp;                              // f padded to 128
    bf16_t* y;                           // down: [rows][d]
    int strips;                          // strips a group
};

// First row of group g: the first `lead` groups hold lead_rows rows each, the offsets
// array counts the others' rows from there.
__device__ __forceinline__ int group_start(const MxArgs& p, int g) {
    return g < p.lead ? g * p.lead_rows : p.lead * p.lead_rows + p.offsets[g - p.lead];
}

__device__ __forceinline__ i32x8 operand(const i32x4& v) {
    return i32x8{v[0], v[1], v[2], v[3], 0, 0, 0, 0};    // 4-bit operands use the lower half
}

// ---------------------------------------------------------------------------
// Strips: groups of few rows, bound by the weight bytes.  A workgroup holds 64 weight rows
// of one group (32 gate rows and the same up rows: 32 hidden columns, one MXFP4 block) over
// all of K, eight waves taking every eighth 128-column step: a weight byte goes from
// memory to the registers of the one wave that multiplies it, no wave waits for another
// before the end, and a row's eight steps in flight are 512 bytes of it.  The waves'
// sums meet in LDS, in wave order.
constexpr int STRIP_WAVES = 8;
constexpr int STRIP_THREADS = STRIP_WAVES * 64;
constexpr int STRIP_ROWS = 64;                           // weight rows
constexpr int STRIP_TILES = STRIP_ROWS / 16;
constexpr int RED_LD = STRIP_ROWS + 4;                   // floats a row of sums in LDS

// MS: 16-row blocks of token rows held at once
template <int MS>
struct StripStep {
    i32x4 b[STRIP_TILES], a[MS];
    uint32_t bs[STRIP_TILES], as[MS];
};

template <bool SWIGLU, int MS>
__global__ __launch_bounds__(STRIP_THREADS, 2) void strip_mxfp4_kernel(MxArgs p) {
    constexpr int BM = 16 * MS;
    constexpr int PARTS = MS == 4 ? 4 : STRIP_WAVES;     // sums in LDS at once (64 KB)
    __shared__ float red[PARTS][BM][RED_LD];
    const int g = blockIdx.x / p.strips, strip = blockIdx.x - g * p.strips;
    const int row0 = group_start(p, g), rows = group_start(p, g + 1) - row0;
    if (rows <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, quarter = lane >> 4;
    const int n0 = strip * (SWIGLU ? STRIP_ROWS / 2 : STRIP_ROWS);
    const int pitch = p.KT * STEP_BYTES;                 // bytes of a row's codes

    // weight rows of the strip: past the matrix's (or, of the gate half, past its N)
    // columns they read as zero; the scale words start at the strip's first row
    const int valid = min(SWIGLU ? STRIP_ROWS / 2 : STRIP_ROWS, p.N - n0);
    auto rsrc = [&](int first) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)(p.w[g] + (int64_t)first * pitch), (short)0,
                                                 max(valid, 0) * pitch, RSRC_WORD3);
    };
    const auto lo = rsrc(n0), hi = rsrc(SWIGLU ? p.N + n0 : n0);
    const uint32_t* wsc = p.ws[g];
    int boff[STRIP_TILES], bsrow[STRIP_TILES];
#pragma unroll
    for (int j = 0; j < STRIP_TILES; ++j) {
        const int r = (SWIGLU && j >= STRIP_TILES / 2 ? j - STRIP_TILES / 2 : j) * 16 + i16;
        boff[j] = r * pitch + quarter * 16;
        // a row past the end has zero codes: any scale of the matrix does
        bsrow[j] = (SWIGLU && j >= STRIP_TILES / 2 ? p.N : 0) + min(n0 + r, p.N - 1);
    }

    for (int m0 = 0; m0 < rows; m0 += BM) {
        // rows past the group repeat its last one; their sums are not stored
        const uint8_t* ap[MS];
        int64_t arow[MS];
#pragma unroll
        for (int m = 0; m < MS; ++m) {
            const int r = row0 + min(m0 + 16 * m + i16, rows - 1);
            arow[m] = p.a_rows ? p.a_rows[r] : r;
            ap[m] = p.a + arow[m] * pitch + quarter * 16;
        }
        f32x4 acc[MS][STRIP_TILES];
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < STRIP_TILES; ++j) acc[m][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto load = [&](StripStep<MS>& s, int t) {
#pragma unroll
            for (int j = 0; j < STRIP_TILES; ++j) {
                s.b[j] = __builtin_bit_cast(
                    i32x4, __builtin_amdgcn_raw_buffer_load_b128(
                               SWIGLU && j >= STRIP_TILES / 2 ? hi : lo, boff[j], t * STEP_BYTES, 0));
                s.bs[j] = wsc[(int64_t)t * p.w_rows + bsrow[j]];
            }
#pragma unroll
            for (int m = 0; m < MS; ++m) {
                s.a[m] = *(const i32x4*)(ap[m] + (int64_t)t * STEP_BYTES);
                s.as[m] = p.as[t * p.a_total + arow[m]];
            }
        };
        // the weights are the matrix instruction's first operand: a lane then holds four
        // consecutive output columns of one row.  A lane's block of 32 is the word's byte
        // `quarter`
        auto multiply = [&](const StripStep<MS>& s) {
            uint32_t sa[MS], sb[STRIP_TILES];
#pragma unroll
            for (int m = 0; m < MS; ++m) sa[m] = s.as[m] >> (8 * quarter);
#pragma unroll
            for (int j = 0; j < STRIP_TILES; ++j) sb[j] = s.bs[j] >> (8 * quarter);
#pragma unroll
            for (int j = 0; j < STRIP_TILES; ++j)
#pragma unroll
                for (int m = 0; m < MS; ++m)
                    acc[m][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                        operand(s.b[j]), operand(s.a[m]), acc[m][j], 4, 4, 0, (int)sb[j], 0,
                        (int)sa[m]);
        };
        // two steps of loads in flight
        StripStep<MS> s0, s1;
        int t = wave;
        if (t < p.KT) load(s0, t);
        if (t + STRIP_WAVES < p.KT) load(s1, t + STRIP_WAVES);
        for (; t < p.KT; t += 2 * STRIP_WAVES) {
            multiply(s0);
            if (t + 2 * STRIP_WAVES < p.KT) load(s0, t + 2 * STRIP_WAVES);
            if (t + STRIP_WAVES < p.KT) {
                multiply(s1);
                if (t + 3 * STRIP_WAVES < p.KT) load(s1, t + 3 * STRIP_WAVES);
            }
        }

        auto at = [&](int part, int m, int j) {
            return (f32x4*)&red[part][16 * m + i16][16 * j + 4 * quarter];
        };
        __syncthreads();                                 // the last row block's sums are read
        if (PARTS < STRIP_WAVES) {
            if (wave >= PARTS)
#pragma unroll
                for (int m = 0; m < MS; ++m)
#pragma unroll
                    for (int j = 0; j < STRIP_TILES; ++j) *at(wave - PARTS, m, j) = acc[m][j];
            __syncthreads();
            if (wave < PARTS)
#pragma unroll
                for (int m = 0; m < MS; ++m)
#pragma unroll
                    for (int j = 0; j < STRIP_TILES; ++j) acc[m][j] += *at(wave, m, j);
            __syncthreads();
        }
        if (wave < PARTS)
#pragma unroll
            for (int m = 0; m < MS; ++m)
#pragma unroll
                for (int j = 0; j < STRIP_TILES; ++j) *at(wave, m, j) = acc[m][j];
        __syncthreads();
        // four output columns a thread
        constexpr int PER_ROW = (SWIGLU ? STRIP_ROWS / 2 : STRIP_ROWS) / 4;
        for (int i = tid; i < BM * PER_ROW; i += STRIP_THREADS) {
            const int r = i / PER_ROW, c = (i % PER_ROW) * 4;
            auto sum = [&](int col) {
                f32x4 v = *(const f32x4*)&red[0][r][col];
#pragma unroll
                for (int q = 1; q < PARTS; ++q) v += *(const f32x4*)&red[q][r][col];
                return v;
            };
            const int row = row0 + m0 + r;
            const bool live = m0 + r < rows;
            if (SWIGLU) {
                const f32x4 a = sum(c), b = sum(STRIP_ROWS / 2 + c);
                float v[4] = {a[0], a[1], a[2], a[3]};
                silu(v);
                uint32_t most = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[e] *= b[e];
                    most = max(most, __float_as_uint(v[e]) & 0x7fffffffu);
                }
                // the block is the eight threads of the row
                most = quad_max(most);
                most = max(most, (uint32_t)__shfl_xor((int)most, 4, 64));
                const uint32_t byte = mx_byte(most);
                const float s = mx_factor(byte);
                uint32_t w = 0;
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * s, v[1] * s, 1.0f, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * s, v[3] * s, 1.0f, 1);
                if (byte == 255u) w = 0;
                if (live) {
                    *(uint16_t*)(p.h + (int64_t)row * (p.hp / 2) + (n0 + c) / 2) = (uint16_t)w;
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
}

template <bool SWIGLU>
int launch_strips(const MxArgs& p, int64_t max_rows, hipStream_t s) {
    const dim3 grid((unsigned)(p.n_groups * p.strips)), block(STRIP_THREADS);
    if (max_rows <= 16)
        hipLaunchKernelGGL((strip_mxfp4_kernel<SWIGLU, 1>), grid, block, 0, s, p);
    else if (max_rows <= 32)
        hipLaunchKernelGGL((strip_mxfp4_kernel<SWIGLU, 2>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((strip_mxfp4_kernel<SWIGLU, 4>), grid, block, 0, s, p);
    return launch_status();
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// workspace: [x codes][x scale words][h codes][h scale words]
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
    int st = launch_quantize_mxfp4_words((const bf16_t*)x, T, d, (uint8_t*)base,
                                         (uint32_t*)(base + at.xs), s);
    if (st != MOE_OK) return st;
    MxArgs p;
    for (int i = 0; i < MOE_MAX_GROUPS; ++i) {
        p.w[i] = i < n_groups ? w13[i] : nullptr;
        p.ws[i] = i < n_groups ? s13[i] : nullptr;
    }
    p.offsets = offsets;
    p.n_groups = n_groups;
    p.lead = lead;
    p.lead_rows = lead_rows;
    p.a = (const uint8_t*)base;
    p.as = (const uint32_t*)(base + at.xs);
    p.a_rows = row_token;
    p.a_total = T;
    p.KT = (int)(mx_cols(d) / 128);
    p.N = f;
    p.w_rows = 2 * f;
    p.h = (uint8_t*)base + at.h;
    p.hs = (uint8_t*)base + at.hs;
    p.h_rows = rows;
    p.hp = (int)mx_cols(f);
    p.y = nullptr;
    p.strips = p.hp / (STRIP_ROWS / 2);
    // a token reaches an expert at most once
    const int64_t max_rows = row_token ? T : rows;
    if ((st = launch_strips<true>(p, max_rows, s)) != MOE_OK) return st;
    for (int i = 0; i < n_groups; ++i) {
        p.w[i] = w2[i];
        p.ws[i] = s2[i];
    }
    p.a = p.h;
    p.as = (const uint32_t*)p.hs;
    p.a_rows = nullptr;
    p.a_total = rows;
    p.KT = p.hp / 128;
    p.N = d;
    p.w_rows = d;
    p.y = (bf16_t*)y;
    p.strips = (int)ceil_div(d, STRIP_ROWS);
    return launch_strips<false>(p, max_rows, s);
}

}  // namespace moe
