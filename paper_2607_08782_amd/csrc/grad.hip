// Gradients around the experts: of the gate-weighted sum (moe_combine_backward) and of the
// gates and gate scores (moe_route_topk_backward).  The gradient of the packaging is the
// combine's sum with weights 1 (combine.hip).  Nothing is added by atomics: every sum has
// one owner and a fixed order.
#include <algorithm>

#include "common.h"
#include "tiles.h"

namespace moe {
namespace {

// Elements as loaded in one 16-byte (V > 1) or one-element chunk.
template <typename Elem, int V>
struct Chunk;
template <>
struct Chunk<bf16_t, 8> {
    uint4 u;
    __device__ __forceinline__ void load(const bf16_t* p) { u = *(const uint4*)p; }
    __device__ __forceinline__ void values(float (&v)[8]) const {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[8]) {
        *(uint4*)p = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
};
template <>
struct Chunk<float, 4> {
    float4 u;
    __device__ __forceinline__ void load(const float* p) { u = *(const float4*)p; }
    __device__ __forceinline__ void values(float (&v)[4]) const {
        v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        *(float4*)p = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <>
struct Chunk<bf16_t, 1> {
    bf16_t u;
    __device__ __forceinline__ void load(const bf16_t* p) { u = *p; }
    __device__ __forceinline__ void values(float (&v)[1]) const { v[0] = bf16_to_f32(u); }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[1]) { *p = f32_to_bf16(v[0]); }
};
template <>
struct Chunk<float, 1> {
    float u;
    __device__ __forceinline__ void load(const float* p) { u = *p; }
    __device__ __forceinline__ void values(float (&v)[1]) const { v[0] = u; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[1]) { *p = v[0]; }
};

// Sum over the wave's lanes, the same order in each; every lane gets it.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// ---------------------------------------------------------------------------
// Gradient of the combine: dy_perm[p] = gate * dy[t] and dgate[t][r] = dy[t] . y_perm[p].
// W waves per token keep the token's dy row in registers (NC chunks a lane; longer rows
// are read again for every assignment) and pass over its local rows: each expert row is
// read and its gradient written once, the dy row read once for all of them.  Bound by the
// memory rate (16384 tokens of Qwen3-30B-A3B: 56 us for 258 MB, 4.6 TB/s).
constexpr int CB_THREADS = 256;

template <typename Elem, int V, int W, int NC>
__global__ __launch_bounds__(CB_THREADS) void combine_backward_kernel(
    const Elem* __restrict__ dy, const Elem* __restrict__ y_perm,
    const int32_t* __restrict__ token_row, const float* __restrict__ gate, int64_t first, int64_t T,
    int d, int k, Elem* __restrict__ dy_perm, float* __restrict__ dgate) {
    __shared__ float part[W > 1 ? MOE_MAX_K : 1][W];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t = (first + blockIdx.x) * (CB_THREADS / 64 / W) + wave / W;
    if (t >= T) return;                                  // whole workgroups where W > 1
    const int sub = wave % W;
    const int chunks = d / V;
    const int per_pass = 64 * W * NC;
    const int rr = lane < k ? lane : k - 1;
    const int p = token_row[t * k + rr];
    const float g = gate ? gate[t * k + rr] : 0.f;
    uint64_t here = __ballot(lane < k && p >= 0);
    Chunk<Elem, V> x[NC];
    auto chunk = [&](int c0, int i) { return c0 + (i * W + sub) * 64 + lane; };
    auto load_dy = [&](int c0) {
#pragma unroll
        for (int i = 0; i < NC; ++i)
            if (chunk(c0, i) < chunks) x[i].load(dy + t * d + (int64_t)chunk(c0, i) * V);
    };
    load_dy(0);
    float mine = 0.f;                                    // lane r: dgate of assignment r
    while (here) {
        const int r = __builtin_ctzll(here);
        here &= here - 1;
        const int64_t row = (int64_t)__builtin_amdgcn_readlane(p, r) * d;
        const float h = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(g), r));
        float dot = 0.f;
        for (int c0 = 0; c0 < chunks; c0 += per_pass) {
            if (chunks > per_pass) load_dy(c0);
            Chunk<Elem, V> y[NC];
            if (dgate)
#pragma unroll
                for (int i = 0; i < NC; ++i)
                    if (chunk(c0, i) < chunks) y[i].load(y_perm + row + (int64_t)chunk(c0, i) * V);
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const int c = chunk(c0, i);
                if (c >= chunks) continue;
                float a[V], b[V];
                x[i].values(a);
                if (dgate) {
                    y[i].values(b);
#pragma unroll
                    for (int j = 0; j < V; ++j) dot = fmaf(a[j], b[j], dot);
                }
                if (dy_perm) {
#pragma unroll
                    for (int j = 0; j < V; ++j) a[j] *= h;
                    Chunk<Elem, V>::store(dy_perm + row + (int64_t)c * V, a);
                }
            }
        }
        if (dgate) {
            dot = wave_sum(dot);
            if (W > 1) {
                if (lane == 0) part[r][sub] = dot;
            }
            mine = lane == r ? dot : mine;
        }
    }
    if (!dgate) return;
    if (W > 1) {
        __syncthreads();
        if (sub == 0 && lane < k) {
            mine = 0.f;
            if (p >= 0)
#pragma unroll
                for (int q = 0; q < W; ++q) mine += part[lane][q];
        }
    }
    if (sub == 0 && lane < k) dgate[t * k + lane] = mine;
}

template <typename Elem, int V>
int combine_backward(const void* dy, const void* y_perm, const int32_t* token_row, const float* gate,
                     int64_t T, int d, int k, void* dy_perm, float* dgate, hipStream_t s) {
    // a wave per token where that fills the chip and a row fits its registers, else four
    const int chunks = d / V;
    const bool wide = T < 4096 || chunks > 64 * 8;
    const int tokens = wide ? 1 : CB_THREADS / 64;       // a workgroup's
    return launch_groups(ceil_div(T, tokens), CB_THREADS, [&](int64_t first, unsigned groups) {
#define MOE_CB(W, NC)                                                                             \
    hipLaunchKernelGGL((combine_backward_kernel<Elem, V, W, NC>), dim3(groups), dim3(CB_THREADS), \
                       0, s, (const Elem*)dy, (const Elem*)y_perm, token_row, gate, first, T, d,  \
                       k, (Elem*)dy_perm, dgate)
        if (wide) {
            if (chunks <= 256) MOE_CB(4, 1);
            else if (chunks <= 512) MOE_CB(4, 2);
            else MOE_CB(4, 4);
        } else {
            if (chunks <= 64) MOE_CB(1, 1);
            else if (chunks <= 128) MOE_CB(1, 2);
            else if (chunks <= 256) MOE_CB(1, 4);
            else MOE_CB(1, 8);
        }
#undef MOE_CB
    });
}

// ---------------------------------------------------------------------------
// Gradient of the gates and gate scores.

// dlogits, a token per wave: four in turn took twice as long where there are few (777 of
// DeepSeek-V2-Lite 7.7 us, this 3.8) and no less where there are many (16384 of Qwen3-30B-A3B
// 9.1 and 8.6).  Lane l holds experts l, l + 64, ...  Beside the dense rows, with MOE_RENORM,
// the chosen experts' values [T][k] (sel).  add (nullable, may be dlogits): what reaches the scores
// another way, added at the end (16384 tokens of 128 experts 8.4 us without and with it); every expert
// then has a gradient, so that dx in fp32 is a dense product (renormalised gates 57 us without, 125 with).
constexpr int RB_THREADS = 256;
constexpr int RJ = MOE_MAX_E / 64;

template <bool RENORM>
__global__ __launch_bounds__(RB_THREADS) void gate_backward_kernel(
    const float* __restrict__ dgate, const float* __restrict__ gate, const int32_t* __restrict__ idx,
    const float* __restrict__ logits, const float* add, int64_t first, int64_t T, int E, int k,
    float* dlogits, float* __restrict__ sel) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t = (first + blockIdx.x) * (RB_THREADS / 64) + wave;
    if (t >= T) return;
    const bool mine = lane < k;
    const int e_r = mine ? idx[t * k + lane] : -1;
    const float p_r = mine ? gate[t * k + lane] : 0.f;
    const float dp_r = mine ? dgate[t * k + lane] : 0.f;
    const float m = wave_sum(p_r * dp_r);
    float v[RJ];
    if (RENORM) {
        const float dl = p_r * (dp_r - m);
        if (sel && mine) sel[t * k + lane] = dl;
#pragma unroll
        for (int j = 0; j < RJ; ++j) v[j] = 0.f;
        for (int r = 0; r < k; ++r) {
            const int e = __builtin_amdgcn_readlane(e_r, r);
            const float x = __uint_as_float(
                (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(dl), r));
#pragma unroll
            for (int j = 0; j < RJ; ++j) v[j] = lane + 64 * j == e ? x : v[j];
        }
    } else {
        float l[RJ], top = -INFINITY, z = 0.f;
#pragma unroll
        for (int j = 0; j < RJ; ++j) {
            l[j] = lane + 64 * j < E ? logits[t * E + lane + 64 * j] : -INFINITY;
            top = fmaxf(top, l[j]);
        }
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
#pragma unroll
        for (int j = 0; j < RJ; ++j) {
            l[j] = expf(l[j] - top);
            z += l[j];
        }
        z = 1.f / wave_sum(z);
        float up[RJ];
#pragma unroll
        for (int j = 0; j < RJ; ++j) up[j] = 0.f;
        for (int r = 0; r < k; ++r) {
            const int e = __builtin_amdgcn_readlane(e_r, r);
            const float x = __uint_as_float(
                (uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(dp_r), r));
#pragma unroll
            for (int j = 0; j < RJ; ++j) up[j] = lane + 64 * j == e ? x : up[j];
        }
#pragma unroll
        for (int j = 0; j < RJ; ++j) v[j] = l[j] * z * (up[j] - m);
    }
#pragma unroll
    for (int j = 0; j < RJ; ++j) {
        if (dlogits && lane + 64 * j < E)
            dlogits[t * E + lane + 64 * j] = add ? v[j] + add[t * E + lane + 64 * j] : v[j];
    }
}

// Four consecutive values of a row of scores from column e on, zero past E; VEC: E is a
// multiple of 4 and rows are 16-byte aligned.
template <bool VEC>
__device__ __forceinline__ f32x4 scores4(const float* row, int e, int E) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (VEC) {
        if (e < E) v = *(const f32x4*)(row + e);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e + i < E) v[i] = row[e + i];
    }
    return v;
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Workgroup b of `total` as (row, column) of a grid of `cols` columns, each XCD (workgroups
// go round-robin over the eight) a contiguous range of it, columns first: the workgroups
// that share rows share an L2, and write whole rows together.
struct Cell {
    int64_t row;
    int col;
};

__device__ __forceinline__ Cell xcd_cell(unsigned b, unsigned total, unsigned cols) {
    const unsigned x = b & 7, q = total >> 3, extra = total & 7;
    const unsigned l = x * q + (x < extra ? x : extra) + (b >> 3);
    return {(int64_t)(l / cols), (int)(l % cols)};
}

// Eight fp32 values as N bf16 terms each (their sum: 8 N significant bits), packed.  What
// remains after a term is exact, and so no term but the last takes more than bf16's largest
// finite value: an infinity, and what would round to one, stays whole in what remains (an
// infinity less itself would make it NaN).
constexpr float BF16_MOST = 0x1.fep127f;

template <int N>
__device__ __forceinline__ void split8(const float (&x)[8], u32x4 (&out)[N]) {
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = r[2 * i], b = r[2 * i + 1];
            if (n + 1 < N) {
                a = __builtin_amdgcn_fmed3f(a, -BF16_MOST, BF16_MOST);
                b = __builtin_amdgcn_fmed3f(b, -BF16_MOST, BF16_MOST);
            }
            const uint32_t w = pack_bf16x2(a, b);
            out[n][i] = w;
            r[2 * i] -= __uint_as_float(w << 16);        // exact
            r[2 * i + 1] -= __uint_as_float(w & 0xffff0000u);
        }
}

// Column c (0..7) of eight rows of eight bf16 values: a matrix operand of eight
// consecutive k, where the rows are k.
__device__ __forceinline__ bf16x8 column(const u32x4 (&row)[8], int c) {
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] = __builtin_amdgcn_perm(row[2 * i + 1][c / 2], row[2 * i][c / 2],
                                     c & 1 ? 0x07060302u : 0x05040100u);
    return __builtin_bit_cast(bf16x8, v);
}

// dw[e][c] = sum_t dlogits[t][e] x[t][c], and dbias.  A wave holds 32 experts x 128 columns.
// Lane (i, q) of it loads, for eight tokens 8 q .. 8 q + 7 of a step of 32, two experts 2 i
// and 2 i + 1 of dlogits and eight columns 8 i .. of x as they lie: its own elements, over
// eight consecutive k, of two operands of the one side and eight of the other (a transpose
// within the lane).  bf16 x: v_mfma_f32_16x16x32_bf16 over dlogits in three bf16 terms, which
// keep all 24 bits, at a third of the rate of the bf16 instruction and five times that of
// the fp32 one, which serves fp32 x.  A step's operands come while the step before
// multiplies.  Eight waves: all blocks of 32 experts (1 to 8), which read x's rows together,
// and tokens among the rest; a workgroup takes one chunk of the tokens, its waves' sums meet
// in LDS in a fixed tree, and the chunks' in sum_parts_kernel in order.  16384 tokens of
// Qwen3-30B-A3B (d = 2048, 128 experts): 31 us and 4 for the sum, where x is 67 MB (13 us);
// with dx in the same launch the matrix units are busy 30 % of the clocks, and the terms and
// transposes take 4.4 vector instructions a matrix one, about as long.  Not kept: x
// through a ring in LDS (36 -> 39 us), a second step of operands in registers (33 -> 34).
constexpr int DW_THREADS = 512;
constexpr int DW_COLS = 128;
constexpr int DW_STEP = 32;
constexpr int DW_EXPERTS = 32;

struct DwArgs {
    const float* dl;
    const void* x;
    int64_t T, chunk;                                    // tokens, tokens per workgroup
    int d, E, eb;                                        // eb: expert blocks (1, 2, 4 or 8)
    int cols;                                            // column tiles
    float* dw;                                           // [chunks][E][d], nullable
    float* dbias;                                        // [chunks][E], nullable
};

typedef f32x4 DwSums[4 * 16 * 64];

template <typename Elem, bool VEC>
__device__ __forceinline__ void router_grad(const DwArgs& p, DwSums& red, unsigned index, unsigned total) {
    constexpr bool BF16 = sizeof(Elem) == 2;
    const int lane = threadIdx.x & 63, i16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int ts_n = 8 / p.eb, block = wave / ts_n, ts = wave % ts_n;
    const Cell cell = xcd_cell(index, total, p.cols);
    const int e0 = block * DW_EXPERTS + 2 * i16, c0 = cell.col * DW_COLS + 8 * i16;
    const int64_t begin = cell.row * p.chunk;
    const int64_t end = begin + p.chunk < p.T ? begin + p.chunk : p.T;
    const bool sums = p.dbias != nullptr && cell.col == 0;
    f32x4 acc[2][8];
    float bias[2] = {0.f, 0.f};
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < 8; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    float2 a[8];
    u32x4 row[8];
    f32x4 wide[BF16 ? 1 : 8][2];                         // fp32 x
    const bool whole = p.d % 4 == 0;                     // rows of 16-byte chunks
    // A step's rows by descriptors that end with the chunk's last token: rows past it, and
    // lanes past the last expert or column, read as zeros (fp32 x: by comparisons).
    constexpr int SIZE = sizeof(Elem);
    auto rsrc = [](const void* base, int bytes) {
        return __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, bytes, RSRC_WORD3);
    };
    __amdgpu_buffer_rsrc_t ra = rsrc(nullptr, 0), rx = ra;
    int64_t at = 0;
    auto seek = [&](int64_t t0) {
        const int rows = t0 < end ? (int)(end - t0 < DW_STEP ? end - t0 : DW_STEP) : 0;
        ra = rsrc(p.dl + t0 * p.E, rows * p.E * 4);
        rx = rsrc((const Elem*)p.x + t0 * p.d, rows * p.d * SIZE);
        at = t0;
    };
    const uint32_t e_stride = (uint32_t)p.E * 4, x_stride = (uint32_t)p.d * SIZE;
    const uint32_t e_off = e0 < p.E ? 8 * quarter * e_stride + 4 * e0 : A_OOB;
    const uint32_t e_off1 = e0 + 1 < p.E ? 8 * quarter * e_stride + 4 * e0 + 4 : A_OOB;
    const uint32_t x_off = c0 < p.d ? 8 * quarter * x_stride + SIZE * c0 : A_OOB;
    auto load = [&](int j) {                             // token at + 8 quarter + j
        if (VEC) {
            a[j] = __builtin_bit_cast(
                float2, __builtin_amdgcn_raw_buffer_load_b64(ra, e_off + j * e_stride, 0, 0));
        } else {
            a[j].x = __uint_as_float(
                __builtin_amdgcn_raw_buffer_load_b32(ra, e_off + j * e_stride, 0, 0));
            a[j].y = __uint_as_float(
                __builtin_amdgcn_raw_buffer_load_b32(ra, e_off1 + j * e_stride, 0, 0));
        }
        if (p.dw == nullptr) return;
        if constexpr (BF16) {
            row[j] = __builtin_bit_cast(
                u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, x_off + j * x_stride, 0, 0));
        } else {
            const bool live = at + 8 * quarter + j < end;
            const float* x = (const float*)p.x + (at + 8 * quarter + j) * p.d;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                wide[j][h] = !live   ? f32x4{0.f, 0.f, 0.f, 0.f}
                             : whole ? scores4<true>(x, c0 + 4 * h, p.d)
                                     : scores4<false>(x, c0 + 4 * h, p.d);
        }
    };
    seek(begin + DW_STEP * ts);
#pragma unroll
    for (int j = 0; j < 8; ++j) load(j);
    for (int64_t t0 = begin + DW_STEP * ts; t0 < end; t0 += DW_STEP * ts_n) {
        seek(t0 + DW_STEP * ts_n);
        if (sums)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                bias[0] += a[j].x;
                bias[1] += a[j].y;
            }
        if constexpr (BF16) {
            float v[2][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[0][j] = a[j].x;
                v[1][j] = a[j].y;
            }
            bf16x8 b[8];
            u32x4 w[2][3];
            if (p.dw != nullptr) {
#pragma unroll
                for (int n = 0; n < 8; ++n) b[n] = column(row, n);
                split8<3>(v[0], w[0]);
                split8<3>(v[1], w[1]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) load(j);
            if (p.dw == nullptr) continue;
            // the small terms first
#pragma unroll
            for (int term = 2; term >= 0; --term)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < 8; ++n)
                        acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, w[m][term]), b[n], acc[m][n], 0, 0, 0);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (p.dw != nullptr)
#pragma unroll
                    for (int m = 0; m < 2; ++m)
#pragma unroll
                        for (int n = 0; n < 8; ++n)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                                m ? a[j].y : a[j].x, wide[j][n / 4][n % 4], acc[m][n], 0, 0, 0);
                load(j);                                 // into the registers just multiplied
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    // token-split waves: the upper half's sums onto the lower half's, until one is left
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        bias[m] += __shfl_xor(bias[m], 16, 64);
        bias[m] += __shfl_xor(bias[m], 32, 64);
    }
    for (int half = ts_n / 2; half >= 1; half /= 2) {
        const int at = block * half + (ts >= half ? ts - half : ts);
        __syncthreads();
        if (ts >= half && ts < 2 * half)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < 8; ++n) red[(at * 16 + m * 8 + n) * 64 + lane] = acc[m][n];
        __syncthreads();
        if (ts < half)
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int n = 0; n < 8; ++n) acc[m][n] += red[(at * 16 + m * 8 + n) * 64 + lane];
        if (!sums) continue;
        float2* rb = (float2*)red;
        __syncthreads();
        if (ts >= half && ts < 2 * half && quarter == 0) rb[at * 16 + i16] = make_float2(bias[0], bias[1]);
        __syncthreads();
        if (ts < half) {
            bias[0] += rb[at * 16 + i16].x;
            bias[1] += rb[at * 16 + i16].y;
        }
    }
    if (ts > 0) return;
    if (sums && quarter == 0)
#pragma unroll
        for (int m = 0; m < 2; ++m)
            if (e0 + m < p.E) p.dbias[cell.row * p.E + e0 + m] = bias[m];
    if (p.dw == nullptr || c0 >= p.d) return;
    // element r of tile (m, n): expert 2 (4 quarter + r) + m of the block, column c0 + n
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int e = block * DW_EXPERTS + 2 * (4 * quarter + r) + m;
            if (e >= p.E) continue;
            float* out = p.dw + (cell.row * p.E + e) * p.d + c0;
            if (BF16 || (whole && c0 + 4 < p.d)) {
                ((f32x4*)out)[0] = f32x4{acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]};
                ((f32x4*)out)[1] = f32x4{acc[m][4][r], acc[m][5][r], acc[m][6][r], acc[m][7][r]};
            } else {
#pragma unroll
                for (int n = 0; n < 8; ++n)
                    if (c0 + n < p.d) out[n] = acc[m][n][r];
            }
        }
}

template <bool VEC>
__global__ __launch_bounds__(DW_THREADS, 2) void router_grad_f32_kernel(DwArgs p) {
    __shared__ DwSums red;
    router_grad<float, VEC>(p, red, blockIdx.x, gridDim.x);
}

// out[i] = sum over n parts of parts[q][i], in order; two such sums in one launch.
struct Parts {
    const float* in;
    float* out;
    int64_t size;
};

__global__ __launch_bounds__(256) void sum_parts_kernel(Parts a, Parts b, int n) {
    int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    Parts p = a;
    if (i >= a.size) {
        i -= a.size;
        p = b;
    }
    if (i >= p.size) return;
    float v = 0.f;
    int q = 0;
    for (; q + 8 <= n; q += 8) {
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = p.in[(q + j) * p.size + i];
#pragma unroll
        for (int j = 0; j < 8; ++j) v += w[j];
    }
    for (; q < n; ++q) v += p.in[q * p.size + i];
    p.out[i] = v;
}

// dx[t][c] = sum_e dlogits[t][e] w[e][c] in bf16.  A wave keeps all experts' rows of w for
// 16 NC columns in registers (KE steps of 32 experts: lane (i, q) loads eight experts 8 q ..
// of a step, NC columns NC i .. each, and transposes them within the lane) and runs over
// blocks of 16 tokens, whose dlogits come, in two bf16 terms (16 bits for an output of 8),
// while the block before multiplies.  Its sums are NC consecutive columns of a row, stored
// at once.  16384 tokens of Qwen3-30B-A3B: 26 us, of which writing dx takes 13 at the rate of
// a copy.
struct DxArgs {
    const float* dlogits;
    const bf16_t* w;
    int64_t T;
    int d, E, runs;                                      // runs: waves side by side over the tokens
    bf16_t* dx;
};

template <int KE, int NC, bool VEC>
__device__ __forceinline__ void scores_backward_bf16(const DxArgs& p, unsigned index, unsigned total) {
    const float* __restrict__ dlogits = p.dlogits;
    const bf16_t* __restrict__ w = p.w;
    bf16_t* __restrict__ dx = p.dx;
    const int64_t T = p.T;
    const int d = p.d, E = p.E, runs = p.runs;
    typedef uint32_t words __attribute__((ext_vector_type(NC / 2)));
    const int lane = threadIdx.x & 63, i16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int cols = (d + 16 * NC - 1) / (16 * NC);
    const Cell cell = xcd_cell(index, total, cols);
    const int c0 = cell.col * 16 * NC + NC * i16;
    bf16x8 b[KE][NC];
#pragma unroll
    for (int s = 0; s < KE; ++s) {
        words row[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = 32 * s + 8 * quarter + j;
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) row[j][i] = 0;
            if (e < E && c0 < d) row[j] = *(const words*)(w + (int64_t)e * d + c0);
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            u32x4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = __builtin_amdgcn_perm(row[2 * i + 1][n / 2], row[2 * i][n / 2],
                                             n & 1 ? 0x07060302u : 0x05040100u);
            b[s][n] = __builtin_bit_cast(bf16x8, v);
        }
    }
    // this wave's token blocks: every runs-th.  Descriptors of a block's rows: rows past T
    // read as zeros and are not stored, nor are columns past d
    const int64_t blocks = (T + 15) / 16;
    auto rsrc = [&](const void* base, int64_t block, int row_bytes) {
        const int rows = block < blocks ? (int)(T - block * 16 < 16 ? T - block * 16 : 16) : 0;
        return __builtin_amdgcn_make_buffer_rsrc((char*)base + block * 16 * row_bytes, (short)0,
                                                 rows * row_bytes, RSRC_WORD3);
    };
    f32x4 lo[KE], hi[KE];
    const int a_off = (i16 * E + 8 * quarter) * 4;
    auto load = [&](int64_t block) {
        const auto r = rsrc(dlogits, block, E * 4);
#pragma unroll
        for (int s = 0; s < KE; ++s) {
            const int e = 32 * s + 8 * quarter;
            if (VEC) {
                lo[s] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                      r, e < E ? a_off + 128 * s : A_OOB, 0, 0));
                hi[s] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                      r, e + 4 < E ? a_off + 128 * s + 16 : A_OOB, 0, 0));
            } else {
                const int64_t t = block * 16 + i16;
                lo[s] = hi[s] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (t < T) {
                    lo[s] = scores4<false>(dlogits + t * E, e, E);
                    hi[s] = scores4<false>(dlogits + t * E, e + 4, E);
                }
            }
        }
    };
    constexpr bool AHEAD = KE <= 4;                      // past 128 experts there is no room
    const uint32_t y_off = c0 < d ? (4 * quarter * d + c0) * 2 : A_OOB;
    int64_t block = cell.row * (DW_THREADS / 64) + wave;
    if (AHEAD) load(block);
    for (; block < blocks; block += runs) {
        u32x4 a[AHEAD ? KE : 1][2];
        auto terms = [&](int s, u32x4 (&out)[2]) {
            const float v[8] = {lo[s][0], lo[s][1], lo[s][2], lo[s][3], hi[s][0], hi[s][1], hi[s][2], hi[s][3]};
            split8<2>(v, out);
        };
        if (AHEAD) {
#pragma unroll
            for (int s = 0; s < KE; ++s) terms(s, a[AHEAD ? s : 0]);
            load(block + runs);
        } else {
            load(block);
        }
        f32x4 acc[NC];
#pragma unroll
        for (int s = 0; s < KE; ++s) {
            if (!AHEAD) {
                __builtin_amdgcn_sched_barrier(0);
                terms(s, a[0]);
            }
#pragma unroll
            for (int term = 1; term >= 0; --term)
#pragma unroll
                for (int n = 0; n < NC; ++n)
                    acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        __builtin_bit_cast(bf16x8, a[AHEAD ? s : 0][term]), b[s][n],
                        s == 0 && term == 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[n], 0, 0, 0);
        }
        const auto ry = rsrc(dx, block, d * 2);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            words v;
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) v[i] = pack_bf16x2(acc[2 * i][r], acc[2 * i + 1][r]);
            if constexpr (NC == 8) __builtin_amdgcn_raw_buffer_store_b128(v, ry, y_off + r * d * 2, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b64(v, ry, y_off + r * d * 2, 0, 0);
        }
    }
}

// Both in one launch, dw's workgroups first: what a short batch saves is a launch (a call of
// 777 tokens of DeepSeek-V2-Lite: 28.5 us with two, 25.5 with one).
template <int KE, int NC, bool VEC>
__global__ __launch_bounds__(DW_THREADS, 2) void router_backward_kernel(DwArgs p, DxArgs q,
                                                                        unsigned dw_groups,
                                                                        unsigned dw_slots) {
    __shared__ DwSums red;
    if (blockIdx.x >= dw_slots)
        scores_backward_bf16<KE, NC, VEC>(q, blockIdx.x - dw_slots, gridDim.x - dw_slots);
    else if (blockIdx.x < dw_groups)
        router_grad<bf16_t, VEC>(p, red, blockIdx.x, dw_groups);
}

// The same in fp32 by v_mfma_f32_16x16x4_f32: 64 tokens x 64 columns a wave, sixteen
// experts a step, of which a lane has four consecutive ones of dlogits' rows and the same
// four rows of w.  8192 tokens of DeepSeek-V2-Lite (64 experts): 38 us, the fp32 matrix
// instruction's 14 and the 13 of writing dx not overlapped.
constexpr int GT = 64;

template <bool VEC>
__global__ __launch_bounds__(256) void scores_backward_f32_kernel(const float* __restrict__ dlogits,
                                                                  const float* __restrict__ w,
                                                                  int first, int64_t T, int d, int E,
                                                                  float* __restrict__ dx) {
    const int lane = threadIdx.x & 63, i16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + wave) * GT;
    const int c0 = (first + (int)blockIdx.y) * GT + 4 * i16;
    if (t0 >= T) return;
    const bool whole = d % 4 == 0;                       // rows of 16-byte chunks
    f32x4 acc[4][4];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int e0 = 0; e0 < E; e0 += 16) {
        const int e = e0 + 4 * quarter;
        f32x4 a[4], b[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int64_t t = t0 + 16 * m + i16;
            a[m] = t < T ? scores4<VEC>(dlogits + t * E, e, E) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const float* row = w + (int64_t)(e + s) * d;
            b[s] = e + s >= E ? f32x4{0.f, 0.f, 0.f, 0.f}
                   : whole    ? scores4<true>(row, c0, d)
                              : scores4<false>(row, c0, d);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n)
                    acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[m][s], b[s][n], acc[m][n], 0, 0, 0);
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t t = t0 + 16 * m + 4 * quarter + r;
            if (t >= T) continue;
            if (whole) {
                if (c0 < d)
                    *(f32x4*)(dx + t * d + c0) = f32x4{acc[m][0][r], acc[m][1][r], acc[m][2][r], acc[m][3][r]};
                continue;
            }
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (c0 + n < d) dx[t * d + c0 + n] = acc[m][n][r];
        }
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// Expert blocks of a dw workgroup, and the chunks of the tokens: a workgroup per CU, two
// steps per wave at least.
int dw_blocks(int E) { return E <= 32 ? 1 : E <= 64 ? 2 : E <= 128 ? 4 : 8; }

struct DwPlan {
    int64_t n, chunk;
    DwPlan(int64_t T, int d, int E) {
        const int64_t step = (int64_t)DW_STEP * (8 / dw_blocks(E));
        const int64_t want = ceil_div(256, ceil_div(d, DW_COLS)), most = ceil_div(T, 2 * step);
        n = std::max<int64_t>(std::min(want, most), 1);
        chunk = ceil_div(ceil_div(T, n), step) * step;
        n = std::max<int64_t>(chunk ? ceil_div(T, chunk) : 1, 1);
    }
};

// workspace: [dlogits when not an output][the chosen experts' values][dw's chunks][dbias']
struct RouteLayout {
    int64_t sel, dw, dbias, total;
    RouteLayout(int64_t T, int d, int E, int k) {
        const int64_t n = DwPlan(T, d, E).n;
        sel = align256(T * E * 4);
        dw = sel + align256(T * k * 4);
        dbias = dw + align256(n * E * d * 4);
        total = dbias + align256(n * E * 4);
    }
};

// dw, dbias (their chunks' sums with plan.n > 1) and dx in bf16; dlogits' rows are those of dl
int launch_router_backward(const float* dl, const float* sel, const int32_t* idx, const void* x,
                           const void* w, int dtype, int64_t T, int d, int E, int k, void* dx,
                           float* dw, float* dbias, float* dw_parts, float* dbias_parts,
                           hipStream_t s) {
    const DwPlan plan(T, d, E);
    const bool sums = dw || dbias;
    DwArgs p;
    p.dl = dl;
    p.x = x;
    p.T = T;
    p.chunk = plan.chunk;
    p.d = d;
    p.E = E;
    p.eb = dw_blocks(E);
    p.dw = !dw ? nullptr : plan.n > 1 ? dw_parts : dw;
    p.dbias = !dbias ? nullptr : plan.n > 1 ? dbias_parts : dbias;
    p.cols = dw ? (int)ceil_div(d, DW_COLS) : 1;
    const unsigned groups = sums ? (unsigned)(p.cols * plan.n) : 0;
    const dim3 block(DW_THREADS);
    const bool vec = E % 4 == 0 && ((uintptr_t)dl & 15u) == 0;
    int st = MOE_OK;
    if (dtype == MOE_BF16) {
        // a workgroup a CU, a block of 16 tokens per wave at least; dw's are rounded to whole
        // rounds over the XCDs
        const unsigned slots = (groups + 7) & ~7u;
        const int64_t cols = ceil_div(d, E > 128 ? 64 : 128), most = ceil_div(ceil_div(T, 16), DW_THREADS / 64);
        const int64_t rows = dx ? std::max<int64_t>(std::min(most, ceil_div(256, cols)), 1) : 0;
        const DxArgs q = {dl, (const bf16_t*)w, T, d, E, (int)(DW_THREADS / 64 * rows), (bf16_t*)dx};
        const dim3 grid((unsigned)(slots + rows * cols));
        if (grid.x == 0) return MOE_OK;
#define MOE_RB(KE, NC, VEC) \
    hipLaunchKernelGGL((router_backward_kernel<KE, NC, VEC>), grid, block, 0, s, p, q, groups, slots)
#define MOE_RB_E(VEC)                   \
    do {                                \
        if (E <= 32) MOE_RB(1, 8, VEC); \
        else if (E <= 64) MOE_RB(2, 8, VEC);  \
        else if (E <= 128) MOE_RB(4, 8, VEC); \
        else MOE_RB(8, 4, VEC);         \
    } while (0)
        if (vec) MOE_RB_E(true);
        else MOE_RB_E(false);
#undef MOE_RB_E
#undef MOE_RB
        st = launch_status();
    } else {
        if (dx && sel) {
            // only the chosen experts' scores have a gradient: their router rows, weighted
            st = launch_combine(w, dtype, idx, sel, nullptr, 0, T, d, k, dx, s);
        } else if (dx) {
            const int cols = (int)ceil_div(d, GT), most = 65535;     // the latter: of a grid
            for (int first = 0; first < cols && st == MOE_OK; first += most) {
                const dim3 grid((unsigned)ceil_div(T, 4 * GT), (unsigned)std::min(cols - first, most));
                if (vec)
                    hipLaunchKernelGGL(scores_backward_f32_kernel<true>, grid, dim3(256), 0, s, dl,
                                       (const float*)w, first, T, d, E, (float*)dx);
                else
                    hipLaunchKernelGGL(scores_backward_f32_kernel<false>, grid, dim3(256), 0, s, dl,
                                       (const float*)w, first, T, d, E, (float*)dx);
                st = launch_status();
            }
        }
        if (st != MOE_OK || !sums) return st;
        if (vec) hipLaunchKernelGGL(router_grad_f32_kernel<true>, dim3(groups), block, 0, s, p);
        else hipLaunchKernelGGL(router_grad_f32_kernel<false>, dim3(groups), block, 0, s, p);
        st = launch_status();
    }
    if (st == MOE_OK && sums && plan.n > 1) {
        const Parts a = {dw_parts, dw, dw ? (int64_t)E * d : 0}, b = {dbias_parts, dbias, dbias ? E : 0};
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)ceil_div(a.size + b.size, 256)), dim3(256), 0,
                           s, a, b, (int)plan.n);
        st = launch_status();
    }
    return st;
}

}  // namespace

int launch_combine_backward(const void* dy, const void* y_perm, int dtype, const int32_t* token_row,
                            const float* gate, int64_t T, int d, int k, void* dy_perm,
                            float* dgate, hipStream_t s) {
    if (T == 0 || (!dy_perm && !dgate)) return MOE_OK;
#define MOE_CB(E, V) \
    combine_backward<E, V>(dy, y_perm, token_row, gate, T, d, k, dy_perm, dgate, s)
    if (dtype == MOE_BF16) return d % 8 == 0 ? MOE_CB(bf16_t, 8) : MOE_CB(bf16_t, 1);
    return d % 4 == 0 ? MOE_CB(float, 4) : MOE_CB(float, 1);
#undef MOE_CB
}

size_t route_backward_ws_bytes(int, int64_t T, int d, int E, int k, int) {
    return (size_t)RouteLayout(T, d, E, k).total + 256;
}

int launch_route_backward(const float* dgate, const float* gate, const int32_t* idx,
                          const float* logits, const float* add, const void* x, const void* w,
                          int dtype, int64_t T, int d, int E, int k, int flags, float* dlogits, void* dx,
                          float* dw, float* dbias, void* ws, hipStream_t s) {
    if (!dlogits && !dx && !dw && !dbias) return MOE_OK;
    const bool renorm = (flags & MOE_RENORM) != 0;
    const RouteLayout at(T, d, E, k);
    char* base = (char*)ws;
    const bool sparse = dx && renorm && dtype == MOE_F32 && !add;
    float* sel = sparse ? (float*)(base + at.sel) : nullptr;
    float* dl = dlogits ? dlogits : dw || dbias || (dx && !sparse) ? (float*)base : nullptr;
    if (T > 0) {
        const int64_t groups = ceil_div(T, RB_THREADS / 64);
        const int st = launch_groups(groups, RB_THREADS, [&](int64_t first, unsigned n) {
            if (renorm)
                hipLaunchKernelGGL(gate_backward_kernel<true>, dim3(n), dim3(RB_THREADS), 0, s, dgate, gate,
                                   idx, logits, add, first, T, E, k, dl, sel);
            else
                hipLaunchKernelGGL(gate_backward_kernel<false>, dim3(n), dim3(RB_THREADS), 0, s, dgate, gate,
                                   idx, logits, add, first, T, E, k, dl, sel);
        });
        if (st != MOE_OK) return st;
    }
    return launch_router_backward(dl, sel, idx, x, w, dtype, T, d, E, k, T > 0 ? dx : nullptr, dw, dbias,
                                  (float*)(base + at.dw), (float*)(base + at.dbias), s);
}

}  // namespace moe
