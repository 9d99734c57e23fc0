// The balance loss of a routing and its gradient (the skew of expert popularity that Sec. III of
// the Director paper finds is what training holds down with it): over the n tokens that count,
// with p[t] = softmax(logits[t]) and c[e] = how often expert e was chosen,
//
//   S[e] = sum_t p[t][e],   loss = E sum_e (c[e] / (k n)) (S[e] / n)
//   dloss / dlogits[t][e] = E / (k n^2) p[t][e] (c[e] - sum_e' p[t][e'] c[e'])
//
// (c is constant: the choice has no gradient.)  Sums have one owner and a fixed order; the counts
// are whole numbers, added by atomics in LDS.
#include <algorithm>

#include "int8.h"

namespace moe {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_GROUPS = 256;                          // parts of the batch

// A value over the L lanes of a token: the same order in each.
template <int L>
__device__ __forceinline__ float token_sum(float v) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o, 64);
    return v;
}

template <int L>
__device__ __forceinline__ float token_max(float v) {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// The softmax of a token's scores, J a lane: lane l of its L holds experts l, l + L, ...
template <int L, int J>
__device__ __forceinline__ void softmax(const float* row, int l, int E, float (&p)[J]) {
    float top = -INFINITY, z = 0.f;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        p[j] = l + L * j < E ? row[l + L * j] : -INFINITY;
        top = fmaxf(top, p[j]);
    }
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

// A group's part of S, of the counts and of n: [groups][E] floats, then ints, then [groups] ints.
struct BalanceParts {
    float* s;
    int32_t* c;
    int32_t* n;
};

BalanceParts parts_at(void* ws, int64_t groups, int E) {
    float* s = (float*)ws;
    int32_t* c = (int32_t*)(s + groups * E);
    return {s, c, c + groups * E};
}

template <int L, int J>
__global__ __launch_bounds__(THREADS) void balance_parts_kernel(const float* __restrict__ logits,
                                                                const int32_t* __restrict__ idx,
                                                                const uint8_t* __restrict__ mask, int64_t T,
                                                                int E, int k, int64_t per, BalanceParts out) {
    constexpr int TOKENS = THREADS / L;                  // at a time
    __shared__ float s[TOKENS][L * J];
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
        softmax<L, J>(logits + t * E, l, E, p);
#pragma unroll
        for (int j = 0; j < J; ++j) sum[j] += p[j];
        for (int r = l; r < k; r += L) {
            const int e = idx[t * k + r];
            if ((unsigned)e < (unsigned)E) atomicAdd(&c[e], 1);
        }
        ++mine;
    }
    if (l == 0 && mine) atomicAdd(&n, mine);
#pragma unroll
    for (int j = 0; j < J; ++j) s[sub][l + L * j] = sum[j];
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += THREADS) {
        float v = 0.f;
        for (int q = 0; q < TOKENS; ++q) v += s[q][e];
        out.s[(int64_t)blockIdx.x * E + e] = v;
        out.c[(int64_t)blockIdx.x * E + e] = c[e];
    }
    if (threadIdx.x == 0) out.n[blockIdx.x] = n;
}

// The parts' sums, and the loss, by one workgroup: 1024 / 256 slices of the parts for each expert.
constexpr int JOIN = 1024;

__global__ __launch_bounds__(JOIN) void balance_join_kernel(BalanceParts in, int groups, int E, int k,
                                                            int32_t* __restrict__ counts,
                                                            float* __restrict__ prob_sum,
                                                            int32_t* __restrict__ n_tokens,
                                                            float* __restrict__ loss) {
    __shared__ double s[JOIN / MOE_MAX_E][MOE_MAX_E], product[JOIN / 64];
    __shared__ int32_t c[JOIN / MOE_MAX_E][MOE_MAX_E];
    __shared__ int64_t tokens[JOIN / 64];
    const int e = threadIdx.x % MOE_MAX_E, slice = threadIdx.x / MOE_MAX_E;
    constexpr int SLICES = JOIN / MOE_MAX_E;
    double v = 0.0;
    int32_t m = 0;
    if (e < E)
        for (int q = slice; q < groups; q += SLICES) {
            v += (double)in.s[(int64_t)q * E + e];
            m += in.c[(int64_t)q * E + e];
        }
    s[slice][e] = v;
    c[slice][e] = m;
    int64_t n = 0;
    for (int q = threadIdx.x; q < groups; q += JOIN) n += in.n[q];
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) n += __shfl_xor(n, o, 64);
    if ((threadIdx.x & 63) == 0) tokens[threadIdx.x >> 6] = n;
    __syncthreads();
    if (slice == 0) {
        for (int q = 1; q < SLICES; ++q) {
            v += s[q][e];
            m += c[q][e];
        }
        if (e < E) {
            counts[e] = m;
            prob_sum[e] = (float)v;
        }
    }
    double x = slice == 0 && e < E ? (double)m * v : 0.0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) product[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x != 0) return;
    n = 0;
    x = 0.0;
    for (int q = 0; q < JOIN / 64; ++q) {
        n += tokens[q];
        x += product[q];
    }
    n_tokens[0] = (int32_t)n;
    loss[0] = n > 0 ? (float)(x * E / ((double)k * (double)n * (double)n)) : 0.f;
}

template <int L, int J>
__global__ __launch_bounds__(THREADS) void balance_backward_kernel(const float* logits,
                                                                   const uint8_t* __restrict__ mask,
                                                                   const int32_t* __restrict__ counts,
                                                                   const int32_t* __restrict__ n_tokens,
                                                                   int64_t T, int E, int k, float scale,
                                                                   float* dlogits) {
    constexpr int TOKENS = THREADS / L;
    const int l = threadIdx.x % L, sub = threadIdx.x / L;
    const double n = (double)max(n_tokens[0], 1);
    const float f = (float)((double)scale * E / ((double)k * n * n));
    // The counts less their mean: the gradient is the same (a token's p sum to 1) and its
    // rounding a matter of how far they spread, not of how large they are.
    int64_t total = 0;
    for (int e = 0; e < E; ++e) total += counts[e];
    const int64_t mean = total / E;
    float c[J];
#pragma unroll
    for (int j = 0; j < J; ++j) c[j] = l + L * j < E ? (float)(counts[l + L * j] - mean) : 0.f;
    for (int64_t t = (int64_t)blockIdx.x * TOKENS + sub; t < T; t += (int64_t)gridDim.x * TOKENS) {
        float p[J];
        const bool live = mask == nullptr || mask[t] != 0;
        if (live) {
            softmax<L, J>(logits + t * E, l, E, p);
            float dot = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j) dot = fmaf(p[j], c[j], dot);
            dot = token_sum<L>(dot);
#pragma unroll
            for (int j = 0; j < J; ++j) p[j] = p[j] * (c[j] - dot) * f;
        }
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (l + L * j < E) dlogits[t * E + l + L * j] = live ? p[j] : 0.f;
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

}  // namespace

// f(L, J) of E experts
#define MOE_LANES(f)             \
    do {                         \
        if (E <= 8) f(8, 1);     \
        else if (E <= 16) f(16, 1); \
        else if (E <= 32) f(32, 1); \
        else if (E <= 64) f(64, 1); \
        else if (E <= 128) f(64, 2); \
        else f(64, 4);           \
    } while (0)

size_t balance_loss_ws_bytes(int64_t T, int E) { return (size_t)(Split(T).groups * (2 * E + 1) * 4) + 256; }

int launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* mask, int64_t T, int E,
                        int k, int32_t* counts, float* prob_sum, int32_t* n_tokens, float* loss,
                        void* ws, hipStream_t s) {
    const Split split(T);
    const BalanceParts parts = parts_at(ws, split.groups, E);
#define MOE_BL(L, J)                                                                             \
    hipLaunchKernelGGL((balance_parts_kernel<L, J>), dim3((unsigned)split.groups), dim3(THREADS), 0, s, \
                       logits, idx, mask, T, E, k, split.per, parts)
    MOE_LANES(MOE_BL);
#undef MOE_BL
    const int st = launch_status();
    if (st != MOE_OK) return st;
    hipLaunchKernelGGL(balance_join_kernel, dim3(1), dim3(JOIN), 0, s, parts, (int)split.groups, E, k, counts,
                       prob_sum, n_tokens, loss);
    return launch_status();
}

int launch_balance_loss_backward(const float* logits, const uint8_t* mask, const int32_t* counts,
                                 const int32_t* n_tokens, int64_t T, int E, int k, float scale,
                                 float* dlogits, hipStream_t s) {
    if (T == 0) return MOE_OK;
#define MOE_BL(L, J)                                                                                  \
    hipLaunchKernelGGL((balance_backward_kernel<L, J>),                                               \
                       dim3((unsigned)std::min<int64_t>(ceil_div(T, THREADS / L), 2048)), dim3(THREADS), 0, s, \
                       logits, mask, counts, n_tokens, T, E, k, scale, dlogits)
    MOE_LANES(MOE_BL);
#undef MOE_BL
    return launch_status();
}

}  // namespace moe
