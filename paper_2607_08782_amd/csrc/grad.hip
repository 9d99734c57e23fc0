// Gradients around the experts: of the gate-weighted sum (moe_combine_backward) and of the
// gates and gate scores (moe_route_topk_backward).  The gradient of the packaging is the
// combine's sum with weights 1 (combine.hip).  Nothing is added by atomics: every sum has
// one owner and a fixed order.
#include "common.h"

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
// memory rate.
constexpr int CB_THREADS = 256;

template <typename Elem, int V, int W, int NC>
__global__ __launch_bounds__(CB_THREADS) void combine_backward_kernel(
    const Elem* __restrict__ dy, const Elem* __restrict__ y_perm,
    const int32_t* __restrict__ token_row, const float* __restrict__ gate, int64_t T, int d, int k,
    Elem* __restrict__ dy_perm, float* __restrict__ dgate) {
    __shared__ float part[W > 1 ? MOE_MAX_K : 1][W];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t = (int64_t)blockIdx.x * (CB_THREADS / 64 / W) + wave / W;
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
#define MOE_CB(W, NC)                                                                            \
    hipLaunchKernelGGL((combine_backward_kernel<Elem, V, W, NC>),                                \
                       dim3((unsigned)ceil_div(T, CB_THREADS / 64 / W)), dim3(CB_THREADS), 0, s, \
                       (const Elem*)dy, (const Elem*)y_perm, token_row, gate, T, d, k,           \
                       (Elem*)dy_perm, dgate)
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
    return launch_status();
}

// ---------------------------------------------------------------------------
// Gradient of the gates and gate scores.

// dlogits of RT tokens a workgroup, a token per wave at a time; lane l holds experts l,
// l + 64, ...  Beside the dense rows, the chosen experts' values [T][k] (sel) and the
// workgroup's column sums (part).
constexpr int RB_THREADS = 256;
constexpr int RT = 16;
constexpr int RJ = MOE_MAX_E / 64;

template <bool RENORM>
__global__ __launch_bounds__(RB_THREADS) void gate_backward_kernel(
    const float* __restrict__ dgate, const float* __restrict__ gate, const int32_t* __restrict__ idx,
    const float* __restrict__ logits, int64_t T, int E, int k, float* __restrict__ dlogits,
    float* __restrict__ sel, float* __restrict__ part) {
    __shared__ float sums[RB_THREADS / 64][MOE_MAX_E];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    float total[RJ] = {};
#pragma unroll
    for (int i = 0; i < RT / (RB_THREADS / 64); ++i) {
        const int64_t t = (int64_t)blockIdx.x * RT + i * (RB_THREADS / 64) + wave;
        if (t >= T) break;
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
            if (dlogits && lane + 64 * j < E) dlogits[t * E + lane + 64 * j] = v[j];
            total[j] += v[j];
        }
    }
    if (!part) return;
#pragma unroll
    for (int j = 0; j < RJ; ++j) sums[wave][lane + 64 * j] = total[j];
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += RB_THREADS) {
        float v = sums[0][e];
#pragma unroll
        for (int q = 1; q < RB_THREADS / 64; ++q) v += sums[q][e];
        part[(int64_t)blockIdx.x * E + e] = v;
    }
}

// Four consecutive values of a row from column c on, zero past `cols`.
template <typename Elem>
__device__ __forceinline__ f32x4 load4(const Elem* row, int c, int cols);
template <>
__device__ __forceinline__ f32x4 load4<float>(const float* row, int c, int cols) {
    f32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < cols ? row[c + i] : 0.f;
    return v;
}
template <>
__device__ __forceinline__ f32x4 load4<bf16_t>(const bf16_t* row, int c, int cols) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (c < cols) {                                      // cols % 8 == 0
        const uint2 u = *(const uint2*)(row + c);
        v = f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u),
                  __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
    }
    return v;
}

// dw[e][c] = sum_t dlogits[t][e] x[t][c] by v_mfma_f32_16x16x4_f32: a wave holds 64 x 64
// of it, the four values a lane loads of a row (experts 4 i .. of dlogits, columns 4 i ..
// of x) being its elements of four operands, so both matrices are read as they lie.  A
// workgroup takes one chunk of the tokens, a quarter of it per wave, summed in LDS.
constexpr int GT = 64;

template <typename Elem>
__global__ __launch_bounds__(256) void router_grad_kernel(const float* __restrict__ dlogits,
                                                          const Elem* __restrict__ x, int64_t T,
                                                          int d, int E, int64_t chunk,
                                                          float* __restrict__ out) {
    __shared__ f32x4 red[3][4][4][64];
    const int lane = threadIdx.x & 63, i16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int c0 = blockIdx.x * GT + 4 * i16, e0 = blockIdx.y * GT + 4 * i16;
    const int64_t begin = (int64_t)blockIdx.z * chunk, end = begin + chunk < T ? begin + chunk : T;
    f32x4 acc[4][4];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    // a step of four tokens, one per quarter
    for (int64_t t0 = begin + 4 * wave; t0 < end; t0 += 16) {
        const int64_t t = t0 + quarter;
        f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
        if (t < end) {
            a = load4<float>(dlogits + t * E, e0, E);
            b = load4<Elem>(x + t * d, c0, d);
        }
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n)
                acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[m], b[n], acc[m][n], 0, 0, 0);
    }
    if (wave > 0)
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n) red[wave - 1][m][n][lane] = acc[m][n];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            // element r of tile (m, n): expert 4 (4 quarter + r) + m, column 4 i16 + n
            const int e = blockIdx.y * GT + 4 * (4 * quarter + r) + m;
            float* row = out + ((int64_t)blockIdx.z * E + e) * d;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const float v = ((acc[m][n][r] + red[0][m][n][lane][r]) + red[1][m][n][lane][r]) +
                                red[2][m][n][lane][r];
                if (e < E && c0 + n < d) row[c0 + n] = v;
            }
        }
}

// dx[t][c] = sum_e dlogits[t][e] w[e][c] by the same instruction: a wave holds 64 tokens x
// 64 columns; sixteen experts a step, of which a lane has four consecutive ones of
// dlogits' rows and the same four rows of w.
template <typename Elem>
__global__ __launch_bounds__(256) void scores_backward_kernel(const float* __restrict__ dlogits,
                                                              const Elem* __restrict__ w, int64_t T,
                                                              int d, int E, Elem* __restrict__ dx) {
    const int lane = threadIdx.x & 63, i16 = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + wave) * GT;
    const int c0 = blockIdx.y * GT + 4 * i16;
    if (t0 >= T) return;
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
            a[m] = t < T ? load4<float>(dlogits + t * E, e, E) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int s = 0; s < 4; ++s)
            b[s] = e + s < E ? load4<Elem>(w + (int64_t)(e + s) * d, c0, d) : f32x4{0.f, 0.f, 0.f, 0.f};
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
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (c0 + n < d) {
                    const float v[1] = {acc[m][n][r]};
                    Chunk<Elem, 1>::store(dx + t * d + c0 + n, v);
                }
        }
}

// out[i] = sum over n parts of parts[q][i], in order.
__global__ __launch_bounds__(256) void sum_parts_kernel(const float* __restrict__ parts, int n,
                                                        int64_t size, float* __restrict__ out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= size) return;
    float v = 0.f;
    for (int q = 0; q < n; ++q) v += parts[q * size + i];
    out[i] = v;
}

int64_t align256(int64_t x) { return (x + 255) & ~(int64_t)255; }

// Token chunks of dw: enough workgroups to fill the chip, 256 tokens each at least.
int64_t grad_chunks(int64_t T, int d, int E) {
    const int64_t tiles = ceil_div(d, GT) * ceil_div(E, GT);
    const int64_t want = ceil_div(512, tiles), most = ceil_div(T, 256);
    const int64_t n = want < most ? want : most;
    return n < 1 ? 1 : n;
}

// workspace: [dlogits when not an output][the chosen experts' values][dw's chunks][dbias'
// parts]
struct RouteLayout {
    int64_t sel, dw, dbias, total;
    RouteLayout(int64_t T, int d, int E, int k) {
        sel = align256(T * E * 4);
        dw = sel + align256(T * k * 4);
        dbias = dw + align256(grad_chunks(T, d, E) * E * d * 4);
        total = dbias + align256(ceil_div(T, RT) * E * 4);
    }
};

template <typename Elem>
int route_products(const float* dl, const float* sel, const int32_t* idx, const void* x, const void* w,
                   int dtype, int64_t T, int d, int E, int k, void* dx, float* dw, float* parts,
                   hipStream_t s) {
    if (dx && sel) {
        // only the chosen experts' scores have a gradient: their router rows, weighted
        const int st = launch_combine(w, dtype, idx, sel, nullptr, 0, T, d, k, dx, s);
        if (st != MOE_OK) return st;
    } else if (dx) {
        hipLaunchKernelGGL((scores_backward_kernel<Elem>),
                           dim3((unsigned)ceil_div(T, 4 * GT), (unsigned)ceil_div(d, GT)), dim3(256),
                           0, s, dl, (const Elem*)w, T, d, E, (Elem*)dx);
    }
    if (dw) {
        const int64_t n = grad_chunks(T, d, E), chunk = ceil_div(ceil_div(T, n), 16) * 16;
        hipLaunchKernelGGL((router_grad_kernel<Elem>),
                           dim3((unsigned)ceil_div(d, GT), (unsigned)ceil_div(E, GT), (unsigned)n),
                           dim3(256), 0, s, dl, (const Elem*)x, T, d, E, chunk, n > 1 ? parts : dw);
        if (n > 1)
            hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)ceil_div((int64_t)E * d, 256)),
                               dim3(256), 0, s, parts, (int)n, (int64_t)E * d, dw);
    }
    return launch_status();
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
                          const float* logits, const void* x, const void* w, int dtype, int64_t T,
                          int d, int E, int k, int flags, float* dlogits, void* dx, float* dw,
                          float* dbias, void* ws, hipStream_t s) {
    if (!dlogits && !dx && !dw && !dbias) return MOE_OK;
    const bool renorm = (flags & MOE_RENORM) != 0;
    const RouteLayout at(T, d, E, k);
    char* base = (char*)ws;
    float* dl = dlogits ? dlogits : dw || (dx && !renorm) ? (float*)base : nullptr;
    float* sel = dx && renorm ? (float*)(base + at.sel) : nullptr;
    float* part = dbias ? (float*)(base + at.dbias) : nullptr;
    if (T > 0) {
        const dim3 grid((unsigned)ceil_div(T, RT)), block(RB_THREADS);
        if (renorm)
            hipLaunchKernelGGL(gate_backward_kernel<true>, grid, block, 0, s, dgate, gate, idx, logits,
                               T, E, k, dl, sel, part);
        else
            hipLaunchKernelGGL(gate_backward_kernel<false>, grid, block, 0, s, dgate, gate, idx,
                               logits, T, E, k, dl, sel, part);
    }
    if (dbias)
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)ceil_div(E, 256)), dim3(256), 0, s, part,
                           (int)ceil_div(T, RT), (int64_t)E, dbias);
    if (T == 0) dx = nullptr;
    float* parts = (float*)(base + at.dw);
    if (dx || dw)
        return dtype == MOE_BF16
                   ? route_products<bf16_t>(dl, sel, idx, x, w, dtype, T, d, E, k, dx, dw, parts, s)
                   : route_products<float>(dl, sel, idx, x, w, dtype, T, d, E, k, dx, dw, parts, s);
    return launch_status();
}

}  // namespace moe
