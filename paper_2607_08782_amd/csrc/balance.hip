// The balance loss of a routing and its gradient (the skew of expert popularity that Sec. III of
// the Director paper finds is what training holds down with it): over the n tokens that count,
// with p[t] = softmax(logits[t]) and c[e] = how often expert e was chosen,
//
//   S[e] = sum_t p[t][e],   loss = E sum_e (c[e] / (k n)) (S[e] / n)
//   dloss / dlogits[t][e] = E / (k n^2) p[t][e] (c[e] - sum_e' p[t][e'] c[e'])
//
// (c is constant: the choice has no gradient.)  Sums have one owner and a fixed order; the counts
// are whole numbers, added by atomics in LDS.
//
// L lanes share a token, so that its scores come in 16-byte loads, side by side, and a softmax needs
// few exchanges.  16384 tokens of 128 experts, 8.4 MB: sums 5.3 us, joining 7.7, gradient 8.0, where the
// bytes of all three are 5.  Joining: eight workgroups, each with 512 parts of 16 experts through one CU, a
// barrier, a wave's sums and a ticket, one after the other.  The gradient, 2.1 TB/s: the tokens' number and
// the counts are read, and divisions in 64 bits done by every lane, before a wave's first product.
#include <algorithm>

#include "int8.h"

namespace moe {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_GROUPS = 512;                          // parts of the batch

// Lane o of the four steps of an exchange within 16 lanes: the quad's neighbour, its other half,
// the other quad of eight lanes, the other eight (data moves within the vector unit; through LDS,
// a shuffle each, the steps of a token took 1.3 us one after the other).
template <int STEP>
__device__ __forceinline__ float other(float v) {
    constexpr int CTRL = STEP == 0 ? 0xb1 : STEP == 1 ? 0x4e : STEP == 2 ? 0x141 : 0x140;
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, false));
}

// A value over the L lanes of a token (2, 4, 8 or 16): the same order in each.
template <int L>
__device__ __forceinline__ float token_sum(float v) {
    v += other<0>(v);
    if (L >= 4) v += other<1>(v);
    if (L >= 8) v += other<2>(v);
    if (L >= 16) v += other<3>(v);
    return v;
}

template <int L>
__device__ __forceinline__ float token_max(float v) {
    v = fmaxf(v, other<0>(v));
    if (L >= 4) v = fmaxf(v, other<1>(v));
    if (L >= 8) v = fmaxf(v, other<2>(v));
    if (L >= 16) v = fmaxf(v, other<3>(v));
    return v;
}

// Expert of a lane's value j: four consecutive ones, then those 4 L further on.
template <int L>
__device__ __forceinline__ int expert_of(int l, int j) {
    return 4 * (l + L * (j / 4)) + j % 4;
}

// A token's scores, 4 C a lane, -infinity past E.  VEC: rows are 16-byte aligned and E % 4 == 0.
template <int L, int C, bool VEC>
__device__ __forceinline__ void load_scores(const float* row, int l, int E, float (&p)[4 * C]) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int e = expert_of<L>(l, 4 * c);
        if (VEC) {
            f32x4 v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (e < E) v = *(const f32x4*)(row + e);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * c + i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * c + i] = e + i < E ? row[e + i] : -INFINITY;
        }
    }
}

// A token's experts, those of a lane, -1 past k (k <= E: with few lanes E is small).
template <int L>
struct Chosen {
    static constexpr int N = L >= 16 ? 1 : L == 8 ? 2 : 4;
    int e[N];
    __device__ __forceinline__ void load(const int32_t* row, int l, int k) {
#pragma unroll
        for (int i = 0; i < N; ++i) e[i] = l + L * i < k ? row[l + L * i] : -1;
    }
    __device__ __forceinline__ void count(int32_t* c, int E) const {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((unsigned)e[i] < (unsigned)E) atomicAdd(&c[e[i]], 1);
    }
};

// The softmax of a token's scores.
template <int L, int J>
__device__ __forceinline__ void softmax(float (&p)[J]) {
    float top = p[0], z = 0.f;
#pragma unroll
    for (int j = 1; j < J; ++j) top = fmaxf(top, p[j]);
    top = token_max<L>(top);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        p[j] = expf(p[j] - top);
        z += p[j];
    }
    z = 1.0f / token_sum<L>(z);
#pragma unroll
    for (int j = 0; j < J; ++j) p[j] *= z;
}

// A group's part of S and of the counts, [groups][E], and of n; the experts' parts of the loss, a
// number each for JOINT experts, and how many of these are there.
struct Part {
    float s;
    int32_t c;
};

constexpr int JOINT = 16;

struct BalanceParts {
    Part* e;
    double* loss;
    int32_t* n;
    uint32_t* ready;
};

BalanceParts parts_at(void* ws, int64_t groups, int E) {
    BalanceParts p;
    p.e = (Part*)ws;
    p.loss = (double*)(p.e + groups * E);
    p.n = (int32_t*)(p.loss + MOE_MAX_E / JOINT);
    p.ready = (uint32_t*)(p.n + groups);
    return p;
}

template <int L, int C, bool VEC>
__global__ __launch_bounds__(THREADS) void balance_parts_kernel(const float* __restrict__ logits,
                                                                const int32_t* __restrict__ idx,
                                                                const uint8_t* __restrict__ mask, int64_t T,
                                                                int E, int k, int64_t per, BalanceParts out) {
    constexpr int TOKENS = THREADS / L, J = 4 * C;       // tokens at a time
    constexpr int JOINED = 16;                           // lanes whose tokens' sums meet in LDS
    __shared__ float s[THREADS / JOINED][L * J];
    __shared__ int32_t c[MOE_MAX_E], n;
    const int l = threadIdx.x % L, sub = threadIdx.x / L;
    for (int e = threadIdx.x; e < E; e += THREADS) c[e] = 0;
    if (threadIdx.x == 0) n = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * per, end = min(begin + per, T);
    float sum[J];
#pragma unroll
    for (int j = 0; j < J; ++j) sum[j] = 0.f;
    int mine = 0;
    for (int64_t t = begin + sub; t < end; t += TOKENS) {
        if (mask != nullptr && mask[t] == 0) continue;   // (all lanes of the token together)
        float p[J];
        Chosen<L> to;
        to.load(idx + t * k, l, k);
        load_scores<L, C, VEC>(logits + t * E, l, E, p);
        to.count(c, E);
        softmax<L>(p);
#pragma unroll
        for (int j = 0; j < J; ++j) sum[j] += p[j];
        ++mine;
    }
    if (l == 0 && mine) atomicAdd(&n, mine);
    // tokens side by side in sixteen lanes first
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (L <= 2) sum[j] += other<1>(sum[j]);
        if (L <= 4) sum[j] += __shfl_xor(sum[j], 4, 64);
        if (L <= 8) sum[j] += __shfl_xor(sum[j], 8, 64);
        if (threadIdx.x % JOINED < L) s[threadIdx.x / JOINED][expert_of<L>(l, j)] = sum[j];
    }
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += THREADS) {
        float v = 0.f;
#pragma unroll
        for (int q = 0; q < THREADS / JOINED; ++q) v += s[q][e];
        out.e[(int64_t)blockIdx.x * E + e] = {v, c[e]};
    }
    if (threadIdx.x == 0) out.n[blockIdx.x] = n;
    if (threadIdx.x == 0 && blockIdx.x == 0) *out.ready = 0;
}

// The parts' sums, by a workgroup for JOINT experts: 64 slices of the parts for each, eight parts in
// flight in a slice.  One workgroup for all experts would read every part through one CU (512 parts
// of 128 experts: 24 us).  The last one to finish adds the experts' parts of the loss, in order.
constexpr int JOIN = 1024;

__global__ __launch_bounds__(JOIN) void balance_join_kernel(BalanceParts in, int groups, int E, int k,
                                                            int32_t* __restrict__ counts,
                                                            float* __restrict__ prob_sum,
                                                            int32_t* __restrict__ n_tokens,
                                                            float* __restrict__ loss) {
    constexpr int SLICES = JOIN / JOINT, AHEAD = 8;
    __shared__ double s[SLICES][JOINT];
    __shared__ int32_t c[SLICES][JOINT];
    __shared__ int64_t tokens[JOIN / 64];
    __shared__ bool last;
    const int col = threadIdx.x % JOINT, e = blockIdx.x * JOINT + col, slice = threadIdx.x / JOINT;
    int64_t n = 0;
    for (int q = threadIdx.x; q < groups; q += JOIN) n += in.n[q];
    double v = 0.0;
    int32_t m = 0;
    if (e < E)
        for (int q0 = slice; q0 < groups; q0 += SLICES * AHEAD) {
            Part a[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                a[i] = q0 + i * SLICES < groups ? in.e[(int64_t)(q0 + i * SLICES) * E + e] : Part{0.f, 0};
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                v += (double)a[i].s;
                m += a[i].c;
            }
        }
    // slices side by side in a wave, then the waves'
#pragma unroll
    for (int o = JOINT; o < 64; o <<= 1) {
        v += __shfl_xor(v, o, 64);
        m += __shfl_xor(m, o, 64);
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o, 64);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) < JOINT) {
        s[wave][col] = v;
        c[wave][col] = m;
    }
    if ((threadIdx.x & 63) == 0) tokens[wave] = n;
    __syncthreads();
    if (wave == 0) {
        v = 0.0;
        m = 0;
#pragma unroll
        for (int q = 0; q < JOIN / 64; ++q) {
            v += s[q][col];
            m += c[q][col];
        }
        if (threadIdx.x < JOINT && e < E) {
            counts[e] = m;
            prob_sum[e] = (float)v;
        }
        double x = e < E ? (double)m * v : 0.0;
#pragma unroll
        for (int o = 1; o < JOINT; o <<= 1) x += __shfl_xor(x, o, 64);
        if (threadIdx.x == 0) {
            __hip_atomic_store(&in.loss[blockIdx.x], x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = __hip_atomic_fetch_add(in.ready, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
        }
    }
    __syncthreads();
    if (!last || threadIdx.x != 0) return;
    n = 0;
    for (int q = 0; q < JOIN / 64; ++q) n += tokens[q];
    double x = 0.0;
    for (unsigned q = 0; q < gridDim.x; ++q)
        x += __hip_atomic_load(&in.loss[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    n_tokens[0] = (int32_t)n;
    loss[0] = n > 0 ? (float)(x * E / ((double)k * (double)n * (double)n)) : 0.f;
}

// A short batch by one workgroup in one launch: the parts are those of its slices, in LDS.  One CU's
// exponentials bound it (loss and gradient of 100 tokens of 60 experts 8.2 us, of 273 10.4, of 777
// 17.7; in two launches 777 take 11).
constexpr int64_t SHORT = 1 << 14;                       // scores

template <int L, int C, bool VEC>
__global__ __launch_bounds__(JOIN) void balance_short_kernel(const float* __restrict__ logits,
                                                             const int32_t* __restrict__ idx,
                                                             const uint8_t* __restrict__ mask, int T, int E,
                                                             int k, int32_t* __restrict__ counts,
                                                             float* __restrict__ prob_sum,
                                                             int32_t* __restrict__ n_tokens,
                                                             float* __restrict__ loss) {
    constexpr int TOKENS = JOIN / L, J = 4 * C, JOINED = 16, AHEAD = C == 1 ? 8 : C == 2 ? 4 : 2;
    __shared__ float s[JOIN / JOINED][L * J];
    __shared__ double product[JOIN / 64];
    __shared__ int32_t c[MOE_MAX_E], n;
    const int l = threadIdx.x % L, sub = threadIdx.x / L;
    for (int e = threadIdx.x; e < E; e += JOIN) c[e] = 0;
    if (threadIdx.x == 0) n = 0;
    __syncthreads();
    float sum[J];
#pragma unroll
    for (int j = 0; j < J; ++j) sum[j] = 0.f;
    int mine = 0;
    for (int t0 = sub; t0 < T; t0 += TOKENS * AHEAD) {   // (all lanes of a token together)
        float p[AHEAD][J];
        Chosen<L> to[AHEAD];
        bool live[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = min(t0 + i * TOKENS, T - 1);
            live[i] = t0 + i * TOKENS < T && (mask == nullptr || mask[t] != 0);
            to[i].load(idx + (int64_t)t * k, l, k);
            load_scores<L, C, VEC>(logits + (int64_t)t * E, l, E, p[i]);
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (!live[i]) continue;
            to[i].count(c, E);
            softmax<L>(p[i]);
#pragma unroll
            for (int j = 0; j < J; ++j) sum[j] += p[i][j];
            ++mine;
        }
    }
    if (l == 0 && mine) atomicAdd(&n, mine);
    // tokens side by side in sixteen lanes first
#pragma unroll
    for (int j = 0; j < J; ++j) {
        if (L <= 2) sum[j] += other<1>(sum[j]);
        if (L <= 4) sum[j] += __shfl_xor(sum[j], 4, 64);
        if (L <= 8) sum[j] += __shfl_xor(sum[j], 8, 64);
        if (threadIdx.x % JOINED < L) s[threadIdx.x / JOINED][expert_of<L>(l, j)] = sum[j];
    }
    __syncthreads();
    const int e = threadIdx.x;
    double x = 0.0;
    if (e < E) {
        double v = 0.0;
#pragma unroll 8
        for (int q = 0; q < JOIN / JOINED; ++q) v += (double)s[q][e];
        counts[e] = c[e];
        prob_sum[e] = (float)v;
        x = (double)c[e] * v;
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) product[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x != 0) return;
    x = 0.0;
    for (int q = 0; q < JOIN / 64; ++q) x += product[q];
    n_tokens[0] = n;
    loss[0] = n > 0 ? (float)(x * E / ((double)k * (double)n * (double)n)) : 0.f;
}

template <int L, int C, bool VEC>
__global__ __launch_bounds__(THREADS) void balance_backward_kernel(const float* logits,
                                                                   const uint8_t* __restrict__ mask,
                                                                   const int32_t* __restrict__ counts,
                                                                   const int32_t* __restrict__ n_tokens,
                                                                   int64_t first, int64_t T, int E, int k,
                                                                   float scale, float* dlogits) {
    constexpr int TOKENS = THREADS / L, J = 4 * C;
    const int l = threadIdx.x % L;
    const int64_t t = (first + blockIdx.x) * TOKENS + threadIdx.x / L;
    if (t >= T) return;                                  // (all lanes of the token together)
    float p[J];
    load_scores<L, C, VEC>(logits + t * E, l, E, p);
    const bool live = mask == nullptr || mask[t] != 0;
    const int64_t n = max(n_tokens[0], 1);
    const float f = (float)((double)scale * E / ((double)k * (double)n * (double)n));
    // The counts less their mean: the gradient is the same (a token's p sum to 1) and its
    // rounding a matter of how far they spread, not of how large they are.
    const int64_t mean = k * n / E;
    float c[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int e = expert_of<L>(l, j);
        c[j] = (float)((e < E ? counts[e] : 0) - mean);
    }
    softmax<L>(p);
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) dot = fmaf(p[j], c[j], dot);
    dot = token_sum<L>(dot);
#pragma unroll
    for (int j = 0; j < J; ++j) p[j] = live ? p[j] * (c[j] - dot) * f : 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const int e = expert_of<L>(l, 4 * i);
        float* out = dlogits + t * E + e;
        if (VEC) {
            if (e < E) *(f32x4*)out = f32x4{p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]};
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (e + j < E) out[j] = p[4 * i + j];
        }
    }
}

// Tokens a group, groups of a batch.
struct Split {
    int64_t per, groups;
    explicit Split(int64_t T) {
        per = std::max<int64_t>(ceil_div(T, MAX_GROUPS), 16);
        groups = std::max<int64_t>(ceil_div(T, per), 1);
    }
};

bool aligned(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace

// f(L, C, VEC) of E experts: lanes of a token, chunks of four experts in each
#define MOE_LANES(f, VEC)                \
    do {                                 \
        if (E <= 8) f(2, 1, VEC);        \
        else if (E <= 16) f(4, 1, VEC);  \
        else if (E <= 32) f(8, 1, VEC);  \
        else if (E <= 64) f(16, 1, VEC); \
        else if (E <= 128) f(16, 2, VEC); \
        else f(16, 4, VEC);              \
    } while (0)

size_t balance_loss_ws_bytes(int64_t T, int E) {
    return (size_t)(Split(T).groups * (2 * E + 1) * 4) + MOE_MAX_E / JOINT * 8 + 256;
}

int launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* mask, int64_t T, int E,
                        int k, int32_t* counts, float* prob_sum, int32_t* n_tokens, float* loss,
                        void* ws, hipStream_t s) {
    const bool vec = E % 4 == 0 && aligned(logits);
    if (T * E <= SHORT) {
#define MOE_BL(L, C, VEC)                                                                              \
    hipLaunchKernelGGL((balance_short_kernel<L, C, VEC>), dim3(1), dim3(JOIN), 0, s, logits, idx, mask, (int)T, \
                       E, k, counts, prob_sum, n_tokens, loss)
        if (vec) MOE_LANES(MOE_BL, true);
        else MOE_LANES(MOE_BL, false);
#undef MOE_BL
        return launch_status();
    }
    const Split split(T);
    const BalanceParts parts = parts_at(ws, split.groups, E);
#define MOE_BL(L, C, VEC)                                                                               \
    hipLaunchKernelGGL((balance_parts_kernel<L, C, VEC>), dim3((unsigned)split.groups), dim3(THREADS), 0, s, \
                       logits, idx, mask, T, E, k, split.per, parts)
    if (vec) MOE_LANES(MOE_BL, true);
    else MOE_LANES(MOE_BL, false);
#undef MOE_BL
    const int st = launch_status();
    if (st != MOE_OK) return st;
    hipLaunchKernelGGL(balance_join_kernel, dim3((unsigned)ceil_div(E, JOINT)), dim3(JOIN), 0, s, parts,
                       (int)split.groups, E, k, counts, prob_sum, n_tokens, loss);
    return launch_status();
}

int launch_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* counts,
                                 const int32_t* n_tokens, int64_t T, int E, int k, float scale,
                                 float* dlogits, hipStream_t s) {
    const bool vec = E % 4 == 0 && aligned(logits) && aligned(dlogits);
    const int lanes = E <= 8 ? 2 : E <= 16 ? 4 : E <= 32 ? 8 : 16;
    return launch_groups(ceil_div(T, THREADS / lanes), THREADS, [&](int64_t first, unsigned groups) {
#define MOE_BL(L, C, VEC)                                                                               \
    hipLaunchKernelGGL((balance_backward_kernel<L, C, VEC>), dim3(groups), dim3(THREADS), 0, s, logits, mask, \
                       counts, n_tokens, first, T, E, k, scale, dlogits)
        if (vec) MOE_LANES(MOE_BL, true);
        else MOE_LANES(MOE_BL, false);
#undef MOE_BL
    });
}

}  // namespace moe
