// Grouped SwiGLU expert FFN in 8-bit integers (Sec. II-A of the Director paper: each expert is an
// FFN sub-network), over ragged groups of rows: token rows and weights in 8 bits, a scale for
// each token and each output channel, both products on the integer matrix instructions, whose
// sums are exact (K up to 2^17: 127 x 127 x 2^17 < 2^31).
//
//   1. h = SiLU(a) b,  a, b = (W1 xq, W3 xq) sx sw, in bf16 (the largest |h| of a row is known
//      only when all of it is; two bytes a value are what the row's way to memory and back takes)
//   2. hq, sh = the rows of h in 8 bits
//   3. y = (W2 hq) sh sw
//
// Rows of codes are padded to whole steps of 128 columns, so no product has a last part of a step.
#include <algorithm>

#include "int8.h"
#include "tiles.h"

namespace moe {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

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
    int strips;                          // strips a group
    int slots;                           // groups that can hold rows at once
};

__device__ __forceinline__ int first_row(const I8Args& p, int g) {
    return group_start(p.offsets, p.lead, p.lead_rows, g);
}

// ---------------------------------------------------------------------------
// Strips: groups of few rows, bound by the weight bytes.  A workgroup holds 16 TILES weight rows
// of one group (of gate/up half gate rows, half the same up rows) over all of K, its W waves
// taking every W-th step: a weight byte goes from memory to the registers of the one wave that
// multiplies it, and no wave waits for another before the end.  The waves' sums meet in LDS.
// MS: 16-row blocks of token rows held at once
template <int MS, int TILES>
struct StripStep {
    i32x4 b[TILES][2], a[MS][2];
};

template <bool SWIGLU, int W, int TILES, int MS, int D>
__device__ __forceinline__ void strip_rows(const I8Args& p, int* red, int g, int n0, int row0, int rows) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int ROWS = 16 * TILES, LD = ROWS + 4, BM = 16 * MS;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int i16 = lane & 15, quarter = lane >> 4;
    const int KT = p.P / STEP;
    // weight rows of the strip: past the matrix's columns (of the gate half, past its N) they
    // read as zero
    const int valid = max(min(SWIGLU ? ROWS / 2 : ROWS, p.N - n0), 0);
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
    for (int m0 = 0; m0 < rows; m0 += BM) {
        // rows past the group repeat its last one; their sums are not stored
        const int8_t* at[MS];
#pragma unroll
        for (int m = 0; m < MS; ++m) {
            const int r = row0 + min(m0 + 16 * m + i16, rows - 1);
            at[m] = p.a + (int64_t)(p.a_rows ? p.a_rows[r] : r) * p.P + quarter * 16;
        }
        i32x4 acc[MS][TILES];
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j) acc[m][j] = i32x4{0, 0, 0, 0};
        // past the end of K: no traffic of the weights, and the last step's rows again
        auto load = [&](StripStep<MS, TILES>& s, int t) {
            const int bytes = t < KT ? valid * p.P - t * STEP : 0;
            const auto lo = rsrc(w_lo + (int64_t)t * STEP, bytes), hi = rsrc(w_hi + (int64_t)t * STEP, bytes);
            const int ta = min(t, KT - 1) * STEP;
#pragma unroll
            for (int j = 0; j < TILES; ++j)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    s.b[j][u] = __builtin_bit_cast(
                        i32x4, __builtin_amdgcn_raw_buffer_load_b128(SWIGLU && j >= TILES / 2 ? hi : lo,
                                                                     boff[j], 64 * u, 0));
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
        for (int i = 0; i < D; ++i) load(s[i], wave + i * W);
        for (int t = wave; t < KT; t += D * W)
#pragma unroll
            for (int i = 0; i < D; ++i) {
                // (past the end: zero weights)
                multiply(s[i]);
                load(s[i], t + (i + D) * W);
            }

        __syncthreads();                                 // the last row block's sums are read
#pragma unroll
        for (int m = 0; m < MS; ++m)
#pragma unroll
            for (int j = 0; j < TILES; ++j)
                *(i32x4*)&red[(wave * BM + 16 * m + i16) * LD + 16 * j + 4 * quarter] = acc[m][j];
        __syncthreads();
        // four output columns a thread
        constexpr int PER_ROW = (SWIGLU ? ROWS / 2 : ROWS) / 4;
        for (int i = tid; i < BM * PER_ROW; i += 64 * W) {
            const int r = i / PER_ROW, c = (i % PER_ROW) * 4;
            if (m0 + r >= rows || n0 + c >= p.N) continue;
            const int row = row0 + m0 + r;
            const float sx = p.as[p.a_rows ? p.a_rows[row] : row];
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
                for (int e = 0; e < 4; ++e) y[e] *= b[e];
            }
            // (h's rows have room past N)
            *(uint2*)(p.out + row * p.pitch + n0 + c) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
        }
    }
#endif
}

// The n-th group that holds rows, its first row and their number (a call of fewer rows than
// groups launches strips for as many groups as it has rows).
struct Group {
    int g, row0, rows;
};

__device__ __forceinline__ Group nth_group(const I8Args& p, int n) {
    const int lane = threadIdx.x & 63;
    for (int g0 = 0; g0 < p.n_groups; g0 += 64) {
        const int g = min(g0 + lane, p.n_groups - 1);
        const int row0 = first_row(p, g), rows = first_row(p, g + 1) - row0;
        uint64_t mask = __ballot(g0 + lane < p.n_groups && rows > 0);
        const int here = __popcll(mask);
        if (n < here) {
            for (; n > 0; --n) mask &= mask - 1;
            const int l = __builtin_ctzll(mask);
            return {g0 + l, __builtin_amdgcn_readlane(row0, l), __builtin_amdgcn_readlane(rows, l)};
        }
        n -= here;
    }
    return {0, 0, 0};
}

// MAX_MS = 1: no group holds more than 16 rows.  Otherwise each group takes the row blocks it needs.
template <bool SWIGLU, int W, int TILES, int MAX_MS>
__global__ __launch_bounds__(64 * W, 2) void strip_int8_kernel(I8Args p) {
    constexpr int SUMS = W * 16 * MAX_MS * (16 * TILES + 4);
    static_assert(SUMS * 4 <= 80 * 1024, "two workgroups share a CU's LDS");
    __shared__ __attribute__((aligned(16))) int red[SUMS];
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
    if (MAX_MS == 1 || of.rows <= 16) strip_rows<SWIGLU, W, TILES, 1, 2>(p, red, of.g, n0, of.row0, of.rows);
    else if (of.rows <= 32) strip_rows<SWIGLU, W, TILES, 2, 2>(p, red, of.g, n0, of.row0, of.rows);
    else strip_rows<SWIGLU, W, TILES, 4, 2>(p, red, of.g, n0, of.row0, of.rows);
}

template <bool SWIGLU>
int launch_strips(I8Args& p, int64_t max_rows, hipStream_t s) {
    constexpr int W = 4, TILES = 4;
    p.strips = (int)ceil_div(SWIGLU ? 2 * (int64_t)p.N : p.N, 16 * TILES);
    const dim3 grid((unsigned)(p.slots * p.strips)), block(64 * W);
    if (max_rows <= 16)
        hipLaunchKernelGGL((strip_int8_kernel<SWIGLU, W, TILES, 1>), grid, block, 0, s, p);
    else
        hipLaunchKernelGGL((strip_int8_kernel<SWIGLU, W, TILES, 4>), grid, block, 0, s, p);
    return launch_status();
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// workspace: [h in bf16][h codes][h scales]
struct Layout {
    int64_t hq, hs, total;
    Layout(int64_t rows, int f) {
        hq = align256(rows * int8_cols(f) * 2);
        hs = hq + align256(rows * int8_cols(f));
        total = hs + align256(rows * 4);
    }
};

}  // namespace

size_t grouped_ffn_int8_ws_bytes(int64_t rows, int f) { return (size_t)Layout(rows, f).total + 256; }

int launch_grouped_ffn_int8(const int8_t* xq, const float* x_scale, int64_t T,
                            const int32_t* row_token, const int32_t* offsets, int n_groups, int lead,
                            int lead_rows, const int8_t* const* w13, const float* const* s13,
                            const int8_t* const* w2, const float* const* s2, int d, int f,
                            int64_t rows, void* y, void* ws, hipStream_t s) {
    if (rows == 0 || T == 0) return MOE_OK;
    const Layout at(rows, f);
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
    p.lead_rows = lead_rows;
    p.a = xq;
    p.as = x_scale;
    p.a_rows = row_token;
    p.P = (int)int8_cols(d);
    p.N = f;
    p.out = (bf16_t*)base;
    p.pitch = int8_cols(f);
    int st = launch_strips<true>(p, max_rows, s);
    if (st != MOE_OK) return st;
    st = launch_quantize_int8(base, MOE_BF16, rows, f, p.pitch, hq, hs, offsets + n_groups - lead,
                              lead * lead_rows, s);
    if (st != MOE_OK) return st;
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
    return launch_strips<false>(p, max_rows, s);
}

}  // namespace moe
