// The norm over all gradients of a step, and their clipping (moe_grad_norm, moe_clip_grads):
// tensors of any number, size and type in few launches.
//
// Every tensor is cut into chunks of CHUNK elements, a workgroup each, numbered over all tensors.
// Squares are summed in 64 bits (no gradient's square overflows or vanishes), a chunk's by its
// threads and their tree, the chunks' in order: the same norm every time.
//
// Bound by the memory rate: 277 MB of fp32 (the matrices of 8 experts of 2048 x 1408) are read for the
// norm in 73 us and read and written to be clipped in 83, where part of them is still in the caches and
// part of what is written goes to memory during the next norm: 5.1 TB/s over both (a copy: 5.4).
// Joining the chunks' sums takes 5.  Chunks of twice the length, last chunks first, and stores past the
// caches were no faster.  81 small tensors, 14 MB in 486 chunks: 6 + 2 + 6 us, where a launch that does little
// takes 2: a workgroup reads its table entry (first, then place, size and type) and then takes two rounds of
// loads, with two workgroups a CU at most to hide them.
#include "int8.h"

namespace moe {
namespace {

constexpr int THREADS = 256;
constexpr int CHUNK = 8192;
constexpr int TABLE = 96;                                // tensors a launch (kernel arguments: 4 KB)

struct Tensors {
    const void* in[TABLE];
    void* out[TABLE];
    int64_t size[TABLE];
    uint32_t first[TABLE];                               // chunks of the launch before the tensor's
    uint8_t dtype[TABLE];
    int n;
};

// The tensor of a workgroup's chunk: the last that starts at or before it.  A wave compares the
// whole table at once (a search's seven loads in turn are longer than a small tensor takes).
__device__ __forceinline__ int tensor_of(const Tensors& t, uint32_t chunk) {
    const int lane = threadIdx.x & 63;
    int n = 0;
#pragma unroll
    for (int i = 0; i < TABLE; i += 64)
        n += __popcll(__ballot(i + lane < t.n && t.first[min(i + lane, TABLE - 1)] <= chunk));
    return __builtin_amdgcn_readfirstlane(n - 1);
}

// A chunk's pieces of a thread, AHEAD of them in flight: f(piece, its place).
constexpr int AHEAD = 4;

template <typename Elem, int V, typename F>
__device__ __forceinline__ void pieces(const Elem* p, int n, const F& f) {
    constexpr int ROUND = THREADS * V;
    int c = threadIdx.x * V;
    for (; c + (AHEAD - 1) * ROUND + V <= n; c += AHEAD * ROUND) {
        Piece<Elem, V> a[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) a[i].load(p + c + i * ROUND);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f(a[i], c + i * ROUND);
    }
    for (; c + V <= n; c += ROUND) {
        Piece<Elem, V> a;
        a.load(p + c);
        f(a, c);
    }
}

template <typename Elem, int V>
__device__ __forceinline__ double squares(const Elem* p, int n) {
    double sum = 0.0;
    auto add = [&](const auto& a) {
        float v[sizeof(a.u) / sizeof(Elem)];
        a.values(v);
#pragma unroll
        for (float x : v) sum = fma((double)x, (double)x, sum);
    };
    pieces<Elem, V>(p, n, [&](const Piece<Elem, V>& a, int) { add(a); });
    if (V > 1 && (int)threadIdx.x < n % V) {             // the last few
        Piece<Elem, 1> a;
        a.load(p + n / V * V + threadIdx.x);
        add(a);
    }
    return sum;
}

__global__ __launch_bounds__(THREADS) void grad_squares_kernel(Tensors t, double* __restrict__ parts) {
    __shared__ double s[THREADS / 64];
    const int i = tensor_of(t, blockIdx.x);
    const int64_t at = (int64_t)(blockIdx.x - t.first[i]) * CHUNK;
    const int n = (int)min(t.size[i] - at, (int64_t)CHUNK);
    const bool whole = ((uintptr_t)t.in[i] & 15u) == 0;
    double sum;
    if (t.dtype[i] == MOE_BF16) {
        const bf16_t* p = (const bf16_t*)t.in[i] + at;
        sum = whole ? squares<bf16_t, 8>(p, n) : squares<bf16_t, 1>(p, n);
    } else {
        const float* p = (const float*)t.in[i] + at;
        sum = whole ? squares<float, 4>(p, n) : squares<float, 1>(p, n);
    }
    sum = lanes_sum(sum);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) parts[blockIdx.x] = (s[0] + s[1]) + (s[2] + s[3]);
}

constexpr int JOIN = 1024;

__global__ __launch_bounds__(JOIN) void grad_norm_kernel(const double* __restrict__ parts, int64_t n,
                                                         float* __restrict__ norm) {
    __shared__ double s[JOIN / 64];
    double sum = 0.0;
    for (int64_t q = threadIdx.x; q < n; q += JOIN) sum += parts[q];
    sum = lanes_sum(sum);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    sum = 0.0;
    for (int q = 0; q < JOIN / 64; ++q) sum += s[q];
    norm[0] = (float)sqrt(sum);
}

// p and out may be the same.
template <typename Elem, int V>
__device__ __forceinline__ void scaled(const Elem* p, Elem* out, int n, float factor) {
    auto put = [&](auto a, int c) {
        float v[sizeof(a.u) / sizeof(Elem)];
        a.values(v);
#pragma unroll
        for (float& x : v) x *= factor;
        a.set(v);
        a.store(out + c);
    };
    pieces<Elem, V>(p, n, [&](const Piece<Elem, V>& a, int c) { put(a, c); });
    if (V > 1 && (int)threadIdx.x < n % V) {
        Piece<Elem, 1> a;
        a.load(p + n / V * V + threadIdx.x);
        put(a, n / V * V + (int)threadIdx.x);
    }
}

__global__ __launch_bounds__(THREADS) void clip_grads_kernel(Tensors t, const float* __restrict__ norm,
                                                             float max_norm) {
    const float now = norm[0];
    const float factor = now <= max_norm ? 1.0f : max_norm / now;
    const int i = tensor_of(t, blockIdx.x);
    if (factor == 1.0f && t.in[i] == t.out[i]) return;   // nothing to change
    const int64_t at = (int64_t)(blockIdx.x - t.first[i]) * CHUNK;
    const int n = (int)min(t.size[i] - at, (int64_t)CHUNK);
    const bool whole = (((uintptr_t)t.in[i] | (uintptr_t)t.out[i]) & 15u) == 0;
    if (t.dtype[i] == MOE_BF16) {
        const bf16_t* p = (const bf16_t*)t.in[i] + at;
        bf16_t* o = (bf16_t*)t.out[i] + at;
        if (whole) scaled<bf16_t, 8>(p, o, n, factor);
        else scaled<bf16_t, 1>(p, o, n, factor);
    } else {
        const float* p = (const float*)t.in[i] + at;
        float* o = (float*)t.out[i] + at;
        if (whole) scaled<float, 4>(p, o, n, factor);
        else scaled<float, 1>(p, o, n, factor);
    }
}

// Launches over tables of up to TABLE tensors and, of these, as many chunks as a grid holds:
// launch(table, groups, chunks before it).
template <typename Launch>
int over_tables(const void* const* in, void* const* out, const int64_t* sizes, const int* dtypes, int n,
                const Launch& launch) {
    Tensors t;
    int64_t before = 0;
    uint64_t chunks = 0;
    t.n = 0;
    auto flush = [&]() {
        if (chunks == 0) return MOE_OK;
        launch(t, (unsigned)chunks, before);
        before += chunks;
        chunks = 0;
        t.n = 0;
        return launch_status();
    };
    constexpr uint64_t MOST = 0xffffffffu / THREADS;     // groups a grid
    for (int i = 0; i < n; ++i) {
        // a tensor longer than a grid goes in pieces
        for (int64_t at = 0; at < sizes[i];) {
            if (t.n == TABLE || chunks == MOST) {
                const int st = flush();
                if (st != MOE_OK) return st;
            }
            const int64_t room = (int64_t)(MOST - chunks) * CHUNK;
            const int64_t take = sizes[i] - at < room ? sizes[i] - at : room;
            const int64_t byte = at * (dtypes[i] == MOE_BF16 ? 2 : 4);
            t.in[t.n] = (const char*)in[i] + byte;
            t.out[t.n] = out ? (char*)out[i] + byte : nullptr;
            t.size[t.n] = take;
            t.first[t.n] = (uint32_t)chunks;
            t.dtype[t.n] = (uint8_t)dtypes[i];
            ++t.n;
            chunks += (uint64_t)ceil_div(take, CHUNK);
            at += take;
        }
    }
    return flush();
}

}  // namespace

int64_t grad_chunks(const int64_t* sizes, int n) {
    int64_t chunks = 0;
    for (int i = 0; i < n; ++i) chunks += ceil_div(sizes[i], CHUNK);
    return chunks;
}

int launch_grad_norm(const void* const* grads, const int64_t* sizes, const int* dtypes, int n,
                     float* norm, void* ws, hipStream_t s) {
    double* parts = (double*)ws;
    const int st = over_tables(grads, nullptr, sizes, dtypes, n, [&](const Tensors& t, unsigned groups, int64_t before) {
        hipLaunchKernelGGL(grad_squares_kernel, dim3(groups), dim3(THREADS), 0, s, t, parts + before);
    });
    if (st != MOE_OK) return st;
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(JOIN), 0, s, parts, grad_chunks(sizes, n), norm);
    return launch_status();
}

int launch_clip_grads(const void* const* grads, const int64_t* sizes, const int* dtypes, int n,
                      const float* norm, float max_norm, void* const* out, hipStream_t s) {
    return over_tables(grads, out, sizes, dtypes, n, [&](const Tensors& t, unsigned groups, int64_t) {
        hipLaunchKernelGGL(clip_grads_kernel, dim3(groups), dim3(THREADS), 0, s, t, norm, max_norm);
    });
}

}  // namespace moe
